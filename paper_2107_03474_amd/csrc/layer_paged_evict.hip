// layer_paged_evict.hip -- part of liblram: eviction from the cache in pages by accumulated attention weight.
//
// Of n keys of a head the `budget` of the highest rank stay: (newest ones first, weight, lowest position) as one 64-bit number
// whose order is theirs, found by a radix selection from the top digit down.  Attention asks for no order of its keys (their
// positions are stored beside them), so only keys that stay and lie past the budget move, into the slots below it that
// are left: n - budget moves at most, and one where a step adds one key.  A workgroup to a head selects, from ranks that it
// keeps in registers; it moves a few keys itself, and leaves many to a second kernel that fills the card.  Bound by the chain of
// dependent steps: 8 us for 256 heads of 2,049 keys, of which one goes; 26 us for 64 heads of 512 to 8,192 keys, many of equal
// weight, and 32 us for the 31,000 keys that move (16 bytes of k and 2 of v lie together, so that a move touches 2 KiB of each).
// Past KEPT ranks a thread a head's workgroup forms them again for every digit: 8 heads of 131,072 keys cut to 4,096 take 453 us,
// and the moves 27, where the ranks' bytes are worth a launch.

#include "layer_paged.h"

namespace {

constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / WAVE;

constexpr int KEPT = 16;        // ranks that a thread keeps: 16,384 of a head; those of the slots behind are formed again
constexpr int MOVED_HERE = 64;  // keys that the selecting workgroup moves itself
constexpr int MOVE_WAVES = 4, MOVE_EACH = 4;  // of the second kernel: waves of a workgroup and keys of a wave (16: 10 us more for 31,000 keys)

struct Evict {
  Pool p;
  int64_t budget, recent;
  int64_t most;    // entries of a list
  int32_t* lists;  // [batch][kv_heads][2][most]: slots that move, and where they go
  int32_t* counts; // [batch][kv_heads]: keys that are left to the second kernel
};

// A slot of no page below the budget counts as taken: nothing can move there.
struct Ranks {
  int64_t newest;
  int budget;
  __device__ __forceinline__ uint64_t operator()(int page, int slot, int position, float weight) const {
    if (page < 0) return slot < budget ? ~(uint64_t)0 : 0;
    const float w = weight + 0.0f;  // -0 is 0
    const uint32_t bits = __builtin_bit_cast(uint32_t, w), up = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    const uint32_t high = position >= newest ? 0xffffffffu : w != w ? 0u : up;
    return (uint64_t)high << 32 | (0x7fffffffu - (uint32_t)position);  // 0x7fffffff - position >= 0
  }
};
__device__ __forceinline__ uint64_t rank_of(const Pool& p, int b, int head, int slot, int64_t newest, int budget) {
  const int page = page_of(p, b, slot);
  const int64_t at = page_rows(p, max(page, 0), head) + (slot & (p.page - 1));
  return Ranks{newest, budget}(page, slot, p.position[at], p.weight[at]);
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

// n <= MOVE_EACH keys of a head on their way to other slots, by a wave: all are read before the first is stored.  Lane i holds
// the place of key i.
template <typename T, int D>
struct Moving {
  using Ti = PageTile<T>;
  using C = typename Chunk<T>::type;
  static constexpr int E = Ti::E, CH = D / E, OF_K = (MOVE_EACH * CH + WAVE - 1) / WAVE, OF_V = MOVE_EACH * D / WAVE;
  C k[OF_K];
  T v[OF_V];
  int position;
  float weight;
  bool has;  // the key lies in a page

  static __device__ __forceinline__ int64_t key_at(int64_t row, int c) {  // pages hold whole blocks, so that a row's place in
    return ((row >> 4 << 4) * D) + (int64_t)(c * 16 + (int)(row & 15)) * E;  // its block is its own
  }
  static __device__ __forceinline__ int64_t value_at(int64_t row, int d) {
    const int r = (int)(row & (Ti::KEYS - 1));
    return (row - r) * D + (int64_t)((d / 16 * 4 + r % 16 / 4) * 16 + d % 16) * E + r / 16 * 4 + r % 4;
  }
  static __device__ __forceinline__ int64_t row_of(const Pool& p, int page, int head, int slot) {
    return page_rows(p, max(page, 0), head) + (slot & (p.page - 1));
  }

  __device__ __forceinline__ void load(const Pool& p, int b, int head, int slot, int n) {
    const int lane = threadIdx.x % WAVE;
    int64_t f = 0;
    has = false;
    if (lane < n) {
      const int page = page_of(p, b, slot);
      has = page >= 0;
      f = row_of(p, page, head, slot);
      position = p.position[f];
      weight = p.weight[f];
    }
#pragma unroll
    for (int j = 0; j < OF_K; ++j) {
      const int i = j * WAVE + lane, key = min(i / CH, MOVE_EACH - 1);
      const int64_t row = __shfl(f, key);
      if (__shfl(has, key) && i < MOVE_EACH * CH) k[j] = *(const C*)((const T*)p.k + key_at(row, i % CH));
    }
#pragma unroll
    for (int j = 0; j < OF_V; ++j) {
      const int i = j * WAVE + lane, key = i / D;
      const int64_t row = __shfl(f, key);
      if (__shfl(has, key)) v[j] = ((const T*)p.v)[value_at(row, i % D)];
    }
  }
  __device__ __forceinline__ void store(const Pool& p, int b, int head, int slot, int n) {
    const int lane = threadIdx.x % WAVE;
    int64_t t = 0;
    if (lane < n) {
      const int page = page_of(p, b, slot);
      has = has && page >= 0;
      t = row_of(p, page, head, slot);
      if (has) {
        p.position[t] = position;
        p.weight[t] = weight;
      }
    }
#pragma unroll
    for (int j = 0; j < OF_K; ++j) {
      const int i = j * WAVE + lane, key = min(i / CH, MOVE_EACH - 1);
      const int64_t row = __shfl(t, key);
      if (__shfl(has, key) && i < MOVE_EACH * CH) *(C*)((T*)p.k + key_at(row, i % CH)) = k[j];
    }
#pragma unroll
    for (int j = 0; j < OF_V; ++j) {
      const int i = j * WAVE + lane, key = i / D;
      const int64_t row = __shfl(t, key);
      if (__shfl(has, key)) ((T*)p.v)[value_at(row, i % D)] = v[j];
    }
  }
};
template <typename T, int D>
__device__ __forceinline__ void move_keys(const Pool& p, int b, int head, const int32_t* from, const int32_t* to, int n) {
  const int i = min((int)threadIdx.x % WAVE, n - 1), f = from[i], t = to[i];
  Moving<T, D> keys;
  keys.load(p, b, head, f, n);
  keys.store(p, b, head, t, n);
}

template <typename T, int D>
__global__ __launch_bounds__(EVICT_THREADS) void k_paged_evict(Evict a) {
  constexpr int BINS = 2048;
  __shared__ int bins[BINS], sums[EVICT_WAVES], chosen[3];
  __shared__ int votes[2][KEPT * EVICT_WAVES];
  __shared__ int32_t near[2][MOVED_HERE];
  const Pool& p = a.p;
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int list = blockIdx.x, head = list % p.kv_heads, b = list / p.kv_heads;
  const int64_t most = p.width << p.log_page;
  const int n = (int)min((int64_t)max(p.used[b], 0), most);
  if (n <= a.budget) {
    if (threadIdx.x == 0) a.counts[list] = 0;
    return;
  }
  const int budget = (int)a.budget;
  const int64_t newest = (int64_t)p.seen[b] - a.recent;
  uint64_t rank[KEPT];
#pragma unroll
  for (int j0 = 0; j0 < KEPT; j0 += 4) {  // four at a time, of the last slot where a thread has none: loads that wait together
    if (j0 * EVICT_THREADS >= n) break;
    int page[4], position[4];
    float weight[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) page[j] = page_of(p, b, min((j0 + j) * EVICT_THREADS + (int)threadIdx.x, n - 1));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int slot = min((j0 + j) * EVICT_THREADS + (int)threadIdx.x, n - 1);
      const int64_t at = page_rows(p, max(page[j], 0), head) + (slot & (p.page - 1));
      position[j] = p.position[at];
      weight[j] = p.weight[at];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      rank[j0 + j] = Ranks{newest, budget}(page[j], (j0 + j) * EVICT_THREADS + (int)threadIdx.x, position[j], weight[j]);
  }
  if (n - budget == 1) {  // a step that adds one key: the lowest rank goes, of equal ones the last
    Moving<T, D> last;  // the key of the last slot, which takes its place, is on its way
    if (wave == 0) last.load(p, b, head, budget, 1);
    uint64_t lowest = ~(uint64_t)0;
    int at = -1;
    const auto look = [&](uint64_t r, int slot) {
      if (r < lowest || (r == lowest && slot > at)) lowest = r, at = slot;
    };
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
      if (j * EVICT_THREADS >= n) break;
      const int slot = j * EVICT_THREADS + threadIdx.x;
      if (slot < n) look(rank[j], slot);
    }
    for (int slot = KEPT * EVICT_THREADS + threadIdx.x; slot < n; slot += EVICT_THREADS)
      look(rank_of(p, b, head, slot, newest, budget), slot);
#pragma unroll
    for (int o = WAVE / 2; o; o /= 2) {
      const uint64_t r = __shfl_xor(lowest, o);
      const int slot = __shfl_xor(at, o);
      look(r, slot);
    }
    __shared__ uint64_t low_rank[EVICT_WAVES];
    if (lane == 0) low_rank[wave] = lowest, sums[wave] = at;
    __syncthreads();
    if (threadIdx.x == 0) a.counts[list] = 0;
    if (wave) return;
    for (int w = 0; w < EVICT_WAVES; ++w) look(low_rank[w], sums[w]);
    if (at < budget) last.store(p, b, head, at, 1);
    return;
  }
  // the digits of the lowest rank that stays, from the top: 11, 11 and 10 bits of either half
  uint64_t mask = 0, prefix = 0;
  int want = budget;  // of the ranks that begin with prefix
  bool all = false;   // these are all there are
  for (int i = 0; i < 6 && !all; ++i) {
    const int shift = i == 0 ? 53 : i == 1 ? 42 : i == 2 ? 32 : i == 3 ? 21 : i == 4 ? 10 : 0;
    const int size = i == 2 || i == 5 ? 1023 : 2047;
    for (int k = threadIdx.x; k < BINS; k += EVICT_THREADS) bins[k] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
      if (j * EVICT_THREADS >= n) break;
      if (j * EVICT_THREADS + (int)threadIdx.x < n && (rank[j] & mask) == prefix) atomicAdd(&bins[rank[j] >> shift & size], 1);
    }
    for (int slot = KEPT * EVICT_THREADS + threadIdx.x; slot < n; slot += EVICT_THREADS) {
      const uint64_t r = rank_of(p, b, head, slot, newest, budget);
      if ((r & mask) == prefix) atomicAdd(&bins[r >> shift & size], 1);
    }
    __syncthreads();
    // thread t: the bins 2047 - 2 t and the one below
    const int high = bins[BINS - 1 - 2 * threadIdx.x], low = bins[BINS - 2 - 2 * threadIdx.x];
    int above = high + low;
#pragma unroll
    for (int o = 1; o < WAVE; o *= 2) {
      const int x = __shfl_up(above, o);
      above += lane >= o ? x : 0;
    }
    if (lane == WAVE - 1) sums[wave] = above;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < EVICT_WAVES; ++w) above += w < wave ? sums[w] : 0;
    above -= high + low;  // of the bins above both
    if (above < want && want <= above + high + low) {  // one thread
      const bool upper = want <= above + high;
      chosen[0] = BINS - 1 - 2 * (int)threadIdx.x - !upper;
      chosen[1] = want - above - (upper ? 0 : high);
      chosen[2] = upper ? high : low;
    }
    __syncthreads();
    prefix |= (uint64_t)chosen[0] << shift;
    mask |= (uint64_t)size << shift;
    want = chosen[1];
    all = want == chosen[2];
  }
  int32_t* const from = a.lists + (int64_t)list * 2 * a.most;
  int32_t* const to = from + a.most;
  const auto put = [&](bool moves, int i, bool hole, int j, int slot) {
    if (moves && i < a.most) from[i] = slot;
    if (hole && j < a.most) to[j] = slot;
    if (moves && i < MOVED_HERE) near[0][i] = slot;
    if (hole && j < MOVED_HERE) near[1][j] = slot;
  };
  int sources = 0, holes = 0, done = 0;
  if (all) {  // every rank that begins with prefix stays: the order of the kept slots in two steps
    uint64_t moving[KEPT], leaving[KEPT];
#pragma unroll
    for (int j = 0; j < KEPT; ++j) {
      const int slot = j * EVICT_THREADS + threadIdx.x;
      const bool stays = slot < n && (rank[j] & mask) >= prefix;
      moving[j] = __builtin_amdgcn_ballot_w64(stays && slot >= budget);
      leaving[j] = __builtin_amdgcn_ballot_w64(!stays && slot < budget);
      if (lane == 0) {
        votes[0][j * EVICT_WAVES + wave] = __popcll(moving[j]);
        votes[1][j * EVICT_WAVES + wave] = __popcll(leaving[j]);
      }
    }
    __syncthreads();
    if (wave < 2) {  // sums of all before, four entries a lane
      static_assert(KEPT * EVICT_WAVES == 4 * WAVE, "four entries a lane");
      int v[4], sum = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) sum += v[k] = votes[wave][lane * 4 + k];
      int up = sum;
#pragma unroll
      for (int o = 1; o < WAVE; o *= 2) {
        const int x = __shfl_up(up, o);
        up += lane >= o ? x : 0;
      }
      if (lane == WAVE - 1) chosen[wave] = up;
      up -= sum;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        votes[wave][lane * 4 + k] = up;
        up += v[k];
      }
    }
    __syncthreads();
    const uint64_t earlier = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < KEPT; ++j)
      put(moving[j] >> lane & 1, votes[0][j * EVICT_WAVES + wave] + __popcll(moving[j] & earlier), leaving[j] >> lane & 1,
          votes[1][j * EVICT_WAVES + wave] + __popcll(leaving[j] & earlier), j * EVICT_THREADS + threadIdx.x);
    sources = chosen[0], holes = chosen[1], done = KEPT * EVICT_THREADS;
  }
  int equal = 0;
  for (int base = done; base < n; base += EVICT_THREADS) {
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
    put(moves, i, hole, j, slot);
  }
  __syncthreads();
  const int count = (int)min((int64_t)min(sources, holes), a.most);
  const bool here = count <= MOVED_HERE;
  if (threadIdx.x == 0) a.counts[list] = here ? 0 : count;
  if (here) {
    constexpr int EACH = MOVED_HERE / EVICT_WAVES;
    static_assert(EACH <= MOVE_EACH, "a wave moves so many at once");
    const int i = wave * EACH;
    if (i < count) move_keys<T, D>(p, b, head, near[0] + i, near[1] + i, min(EACH, count - i));
  }
}

template <typename T, int D>
__global__ __launch_bounds__(MOVE_WAVES* WAVE) void k_paged_move(Evict a, int lists) {
  const int list = blockIdx.x % lists, count = a.counts[list], step = (int)(gridDim.x / lists) * MOVE_WAVES * MOVE_EACH;
  const int32_t* const from = a.lists + (int64_t)list * 2 * a.most;
  for (int i = ((int)(blockIdx.x / lists) * MOVE_WAVES + threadIdx.x / WAVE) * MOVE_EACH; i < count; i += step)
    move_keys<T, D>(a.p, list / a.p.kv_heads, list % a.p.kv_heads, from + i, from + a.most + i, min(count - i, MOVE_EACH));
}

int64_t list_of(const lram_paged& p, int64_t budget) {
  return std::max<int64_t>(0, std::min(budget, p.width * p.page - budget));
}

// Workgroups of the second kernel: no more than fill the card, since a step that moves a few keys leaves it nothing.
constexpr int64_t MOVE_GROUPS = 4096;
int64_t groups_of(const lram_paged& p, int64_t budget) {
  const int64_t most = list_of(p, budget), each = MOVE_WAVES * MOVE_EACH, lists = (int64_t)p.batch * p.kv_heads;
  if (most <= MOVED_HERE || lists == 0) return 0;
  return lists * std::max<int64_t>(1, std::min((most + each - 1) / each, MOVE_GROUPS / lists));
}

size_t workspace_of(const lram_paged& p, int64_t budget) {
  const int64_t most = list_of(p, budget), lists = (int64_t)p.batch * p.kv_heads;
  return most ? (size_t)(lists * (2 * most + 1)) * sizeof(int32_t) : 0;
}

int check_evict(const lram_paged& p, int64_t budget, int64_t recent) {
  if (int rc = check_pool(p, false)) return rc;
  if (budget < 1 || recent < 0 || recent > budget || (p.pages && !p.weight)) return LRAM_EINVAL;
  if ((int64_t)p.batch * p.kv_heads > ((int64_t)1 << 32) / EVICT_THREADS - 1) return LRAM_EINVAL;
  if (groups_of(p, budget) > ((int64_t)1 << 32) / (MOVE_WAVES * WAVE) - 1) return LRAM_EINVAL;
  return LRAM_OK;
}

}  // namespace

extern "C" {

int lram_paged_evict_workspace_bytes(const lram_paged* p, int64_t budget, size_t* bytes) {
  if (!p || !bytes) return LRAM_EINVAL;
  if (int rc = check_evict(*p, budget, 0)) return rc;
  *bytes = workspace_of(*p, budget);
  return LRAM_OK;
}

int lram_paged_evict(const lram_paged* p, int64_t budget, int64_t recent, void* workspace, size_t ws_bytes, void* stream) {
  if (!p) return LRAM_EINVAL;
  if (int rc = check_evict(*p, budget, recent)) return rc;
  Evict a{};
  a.p = pool_of(*p);
  a.budget = budget, a.recent = recent, a.most = list_of(*p, budget);
  if (p->batch == 0 || p->pages == 0 || a.most == 0) return LRAM_OK;  // nothing can be over the budget, or move
  const size_t need = workspace_of(*p, budget);
  if (!workspace || off_align(workspace, 16) || ws_bytes < need) return LRAM_EWORKSPACE;
  const int lists = p->batch * p->kv_heads;
  a.lists = (int32_t*)workspace;
  a.counts = a.lists + (int64_t)lists * 2 * a.most;
  const int64_t groups = groups_of(*p, budget);
  return by_form(p->dtype, p->head_dim, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    hipLaunchKernelGGL((k_paged_evict<T, D>), dim3((unsigned)lists), dim3(EVICT_THREADS), 0, (hipStream_t)stream, a);
    int rc = layer_launched();
    if (rc == LRAM_OK && groups) {
      hipLaunchKernelGGL((k_paged_move<T, D>), dim3((unsigned)groups), dim3(MOVE_WAVES * WAVE), 0, (hipStream_t)stream, a, lists);
      rc = layer_launched();
    }
    return rc;
  });
}

}  // extern "C"
