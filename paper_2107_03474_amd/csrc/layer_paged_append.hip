// layer_paged_append.hip -- part of liblram: new rows into the pages of the cache, and the lengths of its sequences.
//
// Append is one launch.  q: rows rotated as they lie (rotate_chunk).  k: a wave takes the rows of 16 key slots of a sequence and some of
// their heads; a lane owns pairs of 16-byte chunks of single rows and forms their sines and cosines once for all of these
// heads.  v: a wave takes 32 key slots; a lane takes 16 bytes of each of the 4 F keys that lie side by side in the page and
// turns them round in its registers, and a whole block goes out by way of LDS.  Bound by HBM for prompts (28,654 rows of 32/8
// heads of 128 bf16, 704 MB in 145 us, 4.9 TB/s where a large copy reaches 5.1; q and the others in launches of their own took
// 9 us more), by its launch for single tokens (32: 5.5 us).

#include "layer_paged.h"
#include "layer_rotary.h"

namespace {

constexpr int APPEND_WAVES = 4, APPEND_THREADS = APPEND_WAVES * WAVE;

struct Append {
  Pool p;
  Rotate q;  // of q's rows; turns, pairs and magnitude are k's too
  const void *k, *v;
  const float* given;
  int64_t k_row, k_head, v_row, v_head;
  int each;                 // heads that a wave takes
  int64_t places, v_places;  // for tiles of 16 and of 32 slots
  int64_t waves;             // that take v, the first ones (us of 8,200 prompt rows, 16/8 heads of 128: 28, k first 34)
  int64_t groups;            // workgroups that take k and v, the first ones (their way is the longer one); the others take q
};

// Rows of a tile: row t of 16 or 32 is row at + t of the tensors, for from <= t < to, and has position + t.
struct Tile {
  int64_t at;
  int from, to, position;
};

// A chunk into a page.  Pages are next read by other launches, most of them from other L2s, so it goes past the cache (us over two
// sets of data in turn: 28,654 rows of 32/8 heads of 128 bf16 150 -> 145, 8,200 of 16/8 27.2 -> 26.8, keys and values of 32,768
// rows of 8 heads of 64 fp32 68 -> 67; of 128 fp32 it costs, 142 -> 150; one token of 32 sequences is as fast).  Pieces of 64 bytes
// of a lane lose by it (fp32 values of heads of 128: 136 -> 243).
template <typename T>
__device__ __forceinline__ void put(T* to, typename Chunk<T>::type x) {
  __builtin_nontemporal_store(x, (typename Chunk<T>::type*)to);
}

// A lane's chunks of a row, E elements each: units i = lane, lane + 64, ... of 16 rows times D / 2 E pairs of chunks.
template <typename T, int D, Form FORM>
struct Units {
  static constexpr int E = PageTile<T>::E, OF_ROW = D / (2 * E), N = (16 * OF_ROW + WAVE - 1) / WAVE;
  Turn turn[N][E];

  // First elements of unit u's chunks.
  static __device__ __forceinline__ void chunks(const Append& a, int u, int& x, int& y) {
    if (FORM != HALVES || u * E >= a.q.pairs) {
      x = u * 2 * E;
      y = x + E;
    } else {
      x = u * E;
      y = x + a.q.pairs;
    }
  }
  __device__ __forceinline__ void prepare(const Append& a, const Tile& tile) {
    if constexpr (FORM == PLAIN) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = threadIdx.x % WAVE + n * WAVE, t = i / OF_ROW, u = i % OF_ROW;
      if (t < tile.from || t >= tile.to || u * E >= a.q.pairs) continue;
      const int position = tile.position + t;
#pragma unroll
      for (int e = 0; e < E; ++e)
        turn[n][e] = turn_of(a.q.turns[FORM == HALVES ? u * E + e : min(u * E + e, a.q.pairs - 1)], position, a.q.magnitude, 1.0f);
    }
  }
  // Chunks x0 and y0 of unit n rotated.
  using C = Chunk<T>;
  __device__ __forceinline__ void rotate(const Append& a, int n, int u, typename C::type& x0, typename C::type& y0) const {
    if (FORM == PLAIN || u * E >= a.q.pairs) return;
    typename C::wide f = C::up(x0), g = C::up(y0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (FORM == HALVES) {
        const float v = f[e], w = g[e];
        f[e] = fmaf(v, turn[n][e].c, -w * turn[n][e].s);
        g[e] = fmaf(v, turn[n][e].s, w * turn[n][e].c);
      } else {
        typename C::wide& x = e < E / 2 ? f : g;
        const int i = 2 * e % E;
        const bool turns = u * E + e < a.q.pairs;
        const float v = x[i], w = x[i + 1];
        x[i] = turns ? fmaf(v, turn[n][e].c, -w * turn[n][e].s) : v;
        x[i + 1] = turns ? fmaf(v, turn[n][e].s, w * turn[n][e].c) : w;
      }
    }
    x0 = C::down(f);
    y0 = C::down(g);
  }
};

// E elements from e0 on of a row whose halves do not start on a chunk.
template <typename T, int E>
__device__ __forceinline__ typename Chunk<T>::type turned(const Append& a, const T* row, int e0, int position) {
  typename Chunk<T>::wide f = Chunk<T>::up(*(const typename Chunk<T>::type*)(row + e0));
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e0 + e;
    if (i >= 2 * a.q.pairs) break;
    const bool second = i >= a.q.pairs;
    const Turn t = turn_of(a.q.turns[second ? i - a.q.pairs : i], position, a.q.magnitude, 1.0f);
    const float other = (float)row[second ? i - a.q.pairs : i + a.q.pairs];
    f[e] = second ? fmaf(other, t.s, f[e] * t.c) : fmaf(f[e], t.c, -other * t.s);
  }
  return Chunk<T>::down(f);
}

// The chunks of one head of a tile.
template <typename T, int D, Form FORM>
struct Chunks {
  using U = Units<T, D, FORM>;
  typename Chunk<T>::type in[U::N][2];

  __device__ __forceinline__ void load(const Append& a, const Tile& tile, const T* x, int64_t stride) {
#pragma unroll
    for (int n = 0; n < U::N; ++n) {
      const int i = threadIdx.x % WAVE + n * WAVE, t = i / U::OF_ROW;
      int c, d;
      U::chunks(a, i % U::OF_ROW, c, d);
      if (t < tile.from || t >= tile.to) continue;
      in[n][0] = *(const typename Chunk<T>::type*)(x + (tile.at + t) * stride + c);
      in[n][1] = *(const typename Chunk<T>::type*)(x + (tile.at + t) * stride + d);
    }
  }
};

// One head of a tile, rotated, into the page's block.
template <typename T, int D, Form FORM>
__device__ __forceinline__ void turn_head(const Append& a, const Units<T, D, FORM>& units, const Tile& tile, const T* x,
                                          int64_t stride, const Chunks<T, D, FORM>& chunks, T* y) {
  using U = Units<T, D, FORM>;
  constexpr int E = U::E;
  const int lane = threadIdx.x % WAVE;
  const auto place = [](int t, int e0) { return (e0 / E * 16 + t) * E; };  // of the chunk from e0 on of row t
  if constexpr (FORM != ODD_HALVES) {
#pragma unroll
    for (int n = 0; n < U::N; ++n) {
      const int i = lane + n * WAVE, t = i / U::OF_ROW, u = i % U::OF_ROW;
      int c, d;
      U::chunks(a, u, c, d);
      if (t < tile.from || t >= tile.to) continue;
      typename Chunk<T>::type f = chunks.in[n][0], g = chunks.in[n][1];
      units.rotate(a, n, u, f, g);
      put<T>(y + place(t, c), f);
      put<T>(y + place(t, d), g);
    }
  } else {
    for (int i = lane; i < 16 * (D / E); i += WAVE) {
      const int t = i / (D / E), e0 = i % (D / E) * E;
      if (t < tile.from || t >= tile.to) continue;
      put<T>(y + place(t, e0), turned<T, E>(a, x + (tile.at + t) * stride, e0, tile.position + t));
    }
  }
}

// One head of values into a page's block.  In bf16 a whole block goes by way of `lds` (32 rows of the wave's own): a lane's
// 16-byte results lie 128 bytes from the next one's, and go out side by side (28,654 rows of 32/8 heads of 128: 179 -> 146
// us).  In fp32 a lane has 64 bytes in one piece.
template <typename T, int D>
__device__ __forceinline__ void turn_values(const Tile& tile, const T* x, int64_t stride, T* y, typename Chunk<T>::type* lds) {
  using Ti = PageTile<T>;
  constexpr int E = Ti::E, CH = D / E, ITEMS = PAGE_BLOCK * D / (E * E), N = (ITEMS + WAVE - 1) / WAVE;
  const int lane = threadIdx.x % WAVE;
  const bool all = E == 8 && tile.from == 0 && tile.to == PAGE_BLOCK;
  // chunk i of the block, 16 bytes each, spread over the banks
  const auto spread = [](int i) { return i ^ (i >> 6 & 7); };
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = lane + n * WAVE, c = i % CH, g = i / CH % 4, t1 = i / (4 * CH) * Ti::KEYS + 4 * g;
    if (t1 >= PAGE_BLOCK) break;
    typename Chunk<T>::type in[E];
    bool some = false, whole = true;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int t = t1 + e / 4 * 16 + e % 4;
      const bool mine = t >= tile.from && t < tile.to;
      some = some || mine;
      whole = whole && mine;
      if (mine) in[e] = *(const typename Chunk<T>::type*)(x + (tile.at + t) * stride + c * E);
    }
    if (!some) continue;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int d = c * E + j, place = (t1 / Ti::KEYS * (D / 16) + d / 16) * 64 + g * 16 + d % 16;
      typename Chunk<T>::type o;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = in[e][j];
      if (all) {
        lds[spread(place)] = o;
      } else if (whole) {
        *(typename Chunk<T>::type*)(y + place * E) = o;
      } else {
        T* const to = y + place * E;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int t = t1 + e / 4 * 16 + e % 4;
          if (t >= tile.from && t < tile.to) to[e] = o[e];
        }
      }
    }
  }
  if constexpr (E != 8) return;
  if (!all) return;
  wave_lds_sync();  // a lane reads what others wrote
#pragma unroll
  for (int n = 0; n < PAGE_BLOCK * CH / WAVE; ++n)
    put<T>(y + (lane + n * WAVE) * E, lds[spread(lane + n * WAVE)]);
  wave_lds_sync();  // and the next head's block takes its place
}

// Where the tiles of SLOTS slots lie.  Sequence b has the places from start[b] / SLOTS + 2 b on, as many as its n rows can
// need ((n + SLOTS - 2) / SLOTS + 1 tiles), so that a wave finds its own by a search in the starts, 64 at a time.
template <int SLOTS>
struct Places {
  static constexpr int64_t of(int64_t rows, int64_t batch) { return rows / SLOTS + 2 * batch + 1; }
  int b;
  int64_t nth;  // tile of the sequence, negative: none

  __device__ __forceinline__ void find(const Pool& p, int64_t place) {
    const int lane = threadIdx.x % WAVE;
    const auto first = [&](int e) { return clamp_row(p.start[e], p.rows) / SLOTS + 2 * (int64_t)e; };
    int lo = 0, n = p.batch;
    while (n > 1) {
      const int step = (n + WAVE - 1) / WAVE, e = lo + lane * step;
      const uint64_t at = __builtin_amdgcn_ballot_w64(e < lo + n && first(e) <= place);
      const int past = max(__popcll(at) - 1, 0) * step;
      lo += past;
      n = min(step, n - past);
    }
    b = __builtin_amdgcn_readfirstlane(lo);
    nth = p.batch ? place - first(b) : -1;
  }
};

// The rows of a tile that have a slot, from slot `slot` on, of the page `page`.
template <int SLOTS>
__device__ __forceinline__ Tile tile_of(const Pool& p, int64_t place, int& page, int64_t& slot) {
  Places<SLOTS> at;
  at.find(p, place);
  Tile tile{};
  if (at.nth < 0) return tile;
  const CacheSeq s = cache_seq(p, at.b);
  const int64_t first = (int64_t)s.used - (p.start[at.b + 1] - s.q0);  // slot of the row q0
  slot = ((first >> (SLOTS == 16 ? 4 : 5)) + at.nth) * SLOTS;
  if (slot < 0 || slot >= first + s.nq || slot >= s.nk) return tile;
  page = page_of(p, at.b, (int)slot);
  if (page < 0) return tile;
  tile.at = s.q0 + slot - first;
  tile.from = (int)max(first - slot, (int64_t)0);
  tile.to = (int)min(min(first + s.nq, (int64_t)s.nk) - slot, (int64_t)SLOTS);
  tile.position = s.at + (int)(slot - first);
  return tile;
}

// The position of a row, 0 where it belongs to no sequence.
__device__ __forceinline__ int position_of(const Pool& p, int64_t row) {
  int lo = 0, hi = p.batch + 1;  // start[lo - 1] <= row < start[hi]
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (p.start[mid] <= row)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo == 0 || lo > p.batch ? 0 : p.seen[lo - 1] - (int)(p.start[lo] - row);
}

template <typename T, int D, Form FORM>
__global__ __launch_bounds__(APPEND_THREADS) void k_paged_append(Append a) {
  const Pool& p = a.p;
  if constexpr (FORM != PLAIN) {
    if (blockIdx.x >= a.groups) {
      const uint32_t id = (uint32_t)(blockIdx.x - a.groups) * APPEND_THREADS + threadIdx.x;
      const auto position = [&](int64_t row) { return position_of(p, row); };
      if (a.q.past)
        rotate_chunk<T, FORM, true>(a.q, id, position);
      else
        rotate_chunk<T, FORM, false>(a.q, id, position);
      return;
    }
  }
  __shared__ typename Chunk<T>::type lds[APPEND_WAVES][Chunk<T>::E == 8 ? PAGE_BLOCK * D / 8 : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
  int64_t id = (int64_t)blockIdx.x * APPEND_WAVES + wave;
  const bool of_v = id < a.waves;
  if (!of_v) id -= a.waves;
  const int parts = (p.kv_heads + a.each - 1) / a.each;
  const int head0 = (int)(id % parts) * a.each, head1 = min(head0 + a.each, p.kv_heads);
  const int64_t place = id / parts;
  if (place >= (of_v ? a.v_places : a.places)) return;
  int page;
  int64_t slot;
  if (of_v) {
    const Tile tile = tile_of<32>(p, place, page, slot);
    if (tile.from >= tile.to) return;
    for (int head = head0; head < head1; ++head) {
      const int64_t keys = page_rows(p, page, head) + (slot & (p.page - 1));
      turn_values<T, D>(tile, (const T*)a.v + head * a.v_head, a.v_row, (T*)p.v + keys * D, lds[wave]);
    }
    return;
  }
  const Tile tile = tile_of<16>(p, place, page, slot);
  if (tile.from >= tile.to) return;
  // the next head's rows are on their way while one is rotated
  Units<T, D, FORM> units;
  Chunks<T, D, FORM> chunks, next;
  if constexpr (FORM != ODD_HALVES) {
    next.load(a, tile, (const T*)a.k + head0 * a.k_head, a.k_row);
    units.prepare(a, tile);
  }
  for (int head = head0; head < head1; ++head) {
    const T* const rows = (const T*)a.k + head * a.k_head;
    if constexpr (FORM != ODD_HALVES) {
      chunks = next;
      if (head + 1 < head1) next.load(a, tile, rows + a.k_head, a.k_row);
    }
    const int64_t keys = page_rows(p, page, head) + (slot & (p.page - 1));
    turn_head<T, D, FORM>(a, units, tile, rows, a.k_row, chunks, (T*)p.k + keys * D);
    if (lane >= tile.from && lane < tile.to) {
      p.position[keys + lane] = tile.position + lane;
      if (p.weight) p.weight[keys + lane] = a.given ? a.given[(tile.at + lane) * p.kv_heads + head] : 0.0f;
    }
  }
}

// Heads of a wave: as many as leave enough waves to fill the card.
constexpr int KEY_HEADS_EACH = 16;
constexpr int64_t MANY_WAVES = 4096;

constexpr int EXTEND_THREADS = 256;
__global__ __launch_bounds__(EXTEND_THREADS) void k_paged_extend(const int32_t* start, int batch, int32_t* used, int32_t* seen) {
  const int b = blockIdx.x * EXTEND_THREADS + threadIdx.x;
  if (b >= batch) return;
  const int n = max(start[b + 1] - start[b], 0);
  used[b] += n;
  seen[b] += n;
}
__global__ __launch_bounds__(EXTEND_THREADS) void k_paged_shrink(int budget, int batch, int32_t* used) {
  const int b = blockIdx.x * EXTEND_THREADS + threadIdx.x;
  if (b < batch && used[b] > budget) used[b] = budget;
}

}  // namespace

extern "C" {

int lram_paged_extend(const int32_t* start, int32_t batch, int32_t* used, int32_t* seen, void* stream) {
  if (batch < 0 || batch > 1 << 20) return LRAM_EINVAL;
  if (batch == 0) return LRAM_OK;
  if (!start || !used || !seen || off_align(start, 4) || off_align(used, 4) || off_align(seen, 4)) return LRAM_EINVAL;
  hipLaunchKernelGGL(k_paged_extend, dim3((unsigned)((batch + EXTEND_THREADS - 1) / EXTEND_THREADS)), dim3(EXTEND_THREADS), 0,
                     (hipStream_t)stream, start, (int)batch, used, seen);
  return layer_launched();
}

int lram_paged_shrink(int64_t budget, int32_t batch, int32_t* used, void* stream) {
  if (budget < 1 || batch < 0 || batch > 1 << 20) return LRAM_EINVAL;
  if (batch == 0) return LRAM_OK;
  if (!used || off_align(used, 4)) return LRAM_EINVAL;
  hipLaunchKernelGGL(k_paged_shrink, dim3((unsigned)((batch + EXTEND_THREADS - 1) / EXTEND_THREADS)), dim3(EXTEND_THREADS), 0,
                     (hipStream_t)stream, (int)std::min<int64_t>(budget, INT32_MAX), (int)batch, used);
  return layer_launched();
}

int lram_paged_append(const lram_paged* p, const lram_rotary* r, const void* k, int64_t k_row, int64_t k_head,
                      const void* v, int64_t v_row, int64_t v_head, const float* given, const void* q, int64_t q_row,
                      int64_t q_head, void* q_out, void* stream) {
  if (!p) return LRAM_EINVAL;
  if (int rc = check_pool(*p, true)) return rc;
  if (r)
    if (int rc = check_rotary(*r, p->head_dim)) return rc;
  if (bad_strides(k_row, k_head, p->kv_heads, p->head_dim, p->dtype) || bad_strides(v_row, v_head, p->kv_heads, p->head_dim, p->dtype))
    return LRAM_EINVAL;
  if ((q != nullptr) != (q_out != nullptr) || (q && !r) || (given && !p->weight)) return LRAM_EINVAL;
  if (q && (bad_strides(q_row, q_head, p->heads, p->head_dim, p->dtype) || off_align(q, 16) || off_align(q_out, 16)))
    return LRAM_EINVAL;
  if (p->rows == 0) return LRAM_OK;
  if (!k || !v || off_align(k, 16) || off_align(v, 16) || off_align(given, 4)) return LRAM_EINVAL;
  Append a{};
  a.p = pool_of(*p);
  a.k = k, a.v = v, a.given = given;
  a.k_row = k_row, a.k_head = k_head, a.v_row = v_row, a.v_head = v_head;
  a.q.q = q, a.q.q_out = q_out, a.q.q_row = q_row, a.q.q_head = q_head;
  a.q.rows = p->rows, a.q.heads = p->heads, a.q.dim = p->head_dim;
  int64_t q_groups = 0;
  if (r) {
    const int64_t threads = divide(a.q, *r, p->dtype) * p->rows;
    if (q && threads > (int64_t)1 << 31) return LRAM_EINVAL;
    if (q) q_groups = (threads + APPEND_THREADS - 1) / APPEND_THREADS;
  }
  const int64_t most = (((int64_t)1 << 32) / APPEND_THREADS - 1 - q_groups) * APPEND_WAVES;  // a grid: below 2^32 threads
  const auto parts = [&] { return (p->kv_heads + a.each - 1) / a.each; };
  a.places = Places<16>::of(p->rows, p->batch), a.v_places = Places<32>::of(p->rows, p->batch);
  const auto waves = [&] { return (a.places + a.v_places) * parts(); };
  a.each = 1;
  while (a.each < KEY_HEADS_EACH && p->rows / 16 * parts() >= 2 * MANY_WAVES) a.each *= 2;
  while (waves() > most && a.each < p->kv_heads) a.each *= 2;
  if (waves() > most) return LRAM_EINVAL;
  a.waves = a.v_places * parts();
  a.groups = (waves() + APPEND_WAVES - 1) / APPEND_WAVES;
  const int64_t grid = a.groups + q_groups;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(APPEND_THREADS), 0, (hipStream_t)stream, a);
    return layer_launched();
  };
  const Form form = r ? form_of(*r, p->dtype) : PLAIN;
  return by_form(p->dtype, p->head_dim, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return form == PLAIN        ? go(k_paged_append<T, D, PLAIN>)
           : form == NEIGHBOURS ? go(k_paged_append<T, D, NEIGHBOURS>)
           : form == HALVES     ? go(k_paged_append<T, D, HALVES>)
                                : go(k_paged_append<T, D, ODD_HALVES>);
  });
}

}  // extern "C"
