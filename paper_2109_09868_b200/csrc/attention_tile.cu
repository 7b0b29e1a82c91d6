// Attention of several tokens per sequence (prompts, chunks of prompts) over a paged cache, on the tensor cores.
//
// Query rows come in tiles of 128 of one sequence and key head: the query heads that share the key head stand side by side
// (row = token * group + head), so keys and values are read once for all of them.  A CTA walks the tiles of 128 keys that
// any of its rows sees (the sinks' tiles, then the window's), one pass with the running maximum and sum:
//
//   S = Q K^T       128 x 128 fp32 in tensor memory (tcgen05, both operands in shared memory)
//   P = 2^(S' - m)  two threads share a row, 64 scores each in registers; P (bfloat16) goes to tensor memory
//   O += P V        P from tensor memory, V from shared memory as it lies in the cache (MN-major); O fp32 in tensor memory
//
// What a tile's rows wait for is the chain S -> softmax -> P -> O, not any one unit.  Up to D = 64 tensor memory holds S, P
// and O of a tile side by side for two CTAs on an SM: S is free again as soon as it has been loaded into registers, and the
// next one is formed while the softmax works on the last.  Beyond, P lies over S, and the two tiles of a CTA take turns: the
// tensor cores work for one while the other's softmax runs.  The maximum in use is raised, and O rescaled, only when a row's
// grows by more than 2^8 (P and O then still fit their types with room to spare; the final division by the sum makes up
// for it), which after the first tiles is hardly ever.
//
//   8 warps a tile   softmax and output: four for the first 64 keys and columns, four for the others.  Two threads to a row
//                    halve the chain and double the warps that hide it; they need agree on the maximum only when one of
//                    them wants it raised (a vote of the two warps that share rows; the value only then)
//   1 warp           tcgen05.mma for S of one tile; allocates the tensor memory
//   1 warp           tcgen05.mma for O, of two tiles also for S
//   1 warp           tensor-map copies: keys and values by pages, a lane to a page; pages that are not there read as zeros
//   1 warp           looks through the values of tiles that some rows see only in part: a weight of zero must meet no
//                    infinity or NaN, so such elements are taken out, and where a row does see them the output adds them back
//
// Where a call has few query blocks, a cluster of CTAs shares one: each walks a part of the key tiles, and at the end they join
// their rows' maxima, sums and outputs in shared memory, in order.
//
// What bounds it is that chain and its issue, not a unit: at 4,096 causal tokens, D = 128, the tensor cores are busy 48 % of
// the cycles, the special-function unit (a weight is one exponential) 49 %, instructions issue in 43 %.  Measured: 2 x 8,192
// tokens causal, 32 heads on 4 of 128: 925 us, 1,188 TFLOP/s, and 1,080 to 1,100 us, 1,010 TFLOP/s, repeated at the power
// limit; prompts of 1,828 .. 4,096 under a window of 1,024, 32 heads on 8 of 64: 195 to 200 us, 380 TFLOP/s (a CTA lives ten
// steps, four of them masked, and its start and end take the time of three).  Tried and not faster: forming a quarter of the exponentials by a polynomial (the loop's code grows past what the
// instruction caches take well), leaving out the exponentials of keys that no row of a warp sees, one thread to a row, one
// tile to a CTA at D = 128.
#include "async.cuh"

namespace approxifer {

__device__ unsigned int g_attention_tile_wait_timeouts = 0;

namespace {

constexpr int kRows = 128;  // query rows per tile
constexpr int kKeys = 128;  // keys per tile
constexpr int kOtherWarps = 4;
constexpr int kMaxSplit = 8;  // CTAs of a cluster that share a query block
constexpr int kBlock = kRows * 128;  // bytes of 64 columns of a tile
constexpr float kGrowth = 8.f;       // log2 of what the maximum in use may lag behind

constexpr int tile_bytes(int dp) { return kBlock * (dp / 64); }
// Query tiles per CTA and CTAs per SM.  Up to D = 64 a CTA has one tile and two CTAs share an SM: each fills the gaps of the
// other, its start and end included.  Beyond, shared memory holds one CTA, and its two tiles share the keys and values.
constexpr int tiles_of(int dp) { return dp == 64 ? 1 : 2; }
constexpr int threads_of(int dp) { return (8 * tiles_of(dp) + kOtherWarps) * 32; }
constexpr int kStages = 5;
// Rings of one entry per tile of keys.  The copies go in order through kStages places, so that the values of tile j + 4, or
// the keys of tile j + 8, are asked for only after those of tile j have been used and given back.
constexpr int kCleans = 4, kMasks = 8;
// The ring's entries are keys and values in turn: entry 2j the keys of tile j, 2j + 1 its values, entry i in place i % kStages.  A
// place thus holds both kinds in turn, but the warps that look through the values, or form S, wait for one kind only.  A wait by
// parity tells two phases apart, no more: on a barrier that both kinds used, such a warp could take the entry before the last for
// the last while the one between, which it never asks for, is still on its way.  So a place has two barriers for what has landed,
// one for each kind, and who waits on one has waited for each of its phases.  (The products with the values wait for the look
// through them, which has waited for the values: a wait of their own for the values too cost 6 % of the windowed prompts.)
constexpr int kFulls = 2 * kStages;
static_assert(kStages % 2 == 1, "a place holds keys and values in turn");
// alignment, barriers and flags, what the threads of a row exchange, queries, ring
constexpr int smem_bytes(int dp) { return 1024 + 1024 + tiles_of(dp) * kRows * 4 + (tiles_of(dp) + kStages) * tile_bytes(dp); }

struct TileArgs {
  approxifer_attention_args a;
  int32_t group, tokens;  // query heads per key head; tokens per tile (128 / group)
  int32_t blocks;         // query blocks (a CTA's tiles) per sequence
  int32_t page_shift;
};

// What the CTA works on; all roles derive it alike.
struct Job {
  int b, hk, token0;   // first token (in the packed array)
  int left;            // tokens of the sequence from there on
  int pos0;            // position of the first token (may be negative: fewer cached tokens than queries)
  int lo, p1;          // lowest position in a window, highest position seen
  int window, sinks;
  int tokens;          // per tile
  int sink_tiles, first_tile;
  int skip, steps;       // this CTA's steps of the cluster's: from `skip` on
  int steps0, steps1;  // of the two query tiles

  __device__ __forceinline__ int tile(int j) const { return j + skip < sink_tiles ? j + skip : first_tile + (j + skip - sink_tiles); }
  __device__ __forceinline__ int first_pos(int t) const { return pos0 + t * tokens; }
  __device__ __forceinline__ int last_pos(int t) const { return pos0 + min((t + 1) * tokens, left) - 1; }
  // Which steps a query tile takes part in: tile 0 up to the last key its rows see, tile 1 all (the window of its first row
  // may start a tile or two later than tile 0's; there it finds nothing).
  __device__ __forceinline__ int steps_of(int t) const { return t == 0 ? steps0 : steps1; }
  // which of the 32 keys from position k on the row at `pos` sees, a bit per key
  __device__ __forceinline__ uint32_t sees(int pos, int k) const {
    auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };  // bits 0 .. n-1
    const uint32_t past = below(pos + 1 - k);
    return window == 0 ? past : past & (~below(pos + 1 - window - k) | below(sinks - k));
  }
  __device__ __forceinline__ bool full(int t, int j) const {
    const int k0 = tile(j) * kKeys, k1 = k0 + kKeys - 1;
    return k1 <= first_pos(t) && (window == 0 || k0 > last_pos(t) - window || k1 < sinks);
  }
  // steps from `from` up to `to` are full for query tile t (tiles that hold sinks are left to the masked way)
  __device__ __forceinline__ void full_steps(int t, int* from, int* to) const {
    const int past = last_pos(t) - window, k0 = window && past >= 0 ? past / kKeys + 1 : 0, k1 = first_pos(t) < 0 ? 0 : (first_pos(t) + 1) / kKeys;
    *from = sink_tiles + max(0, k0 - first_tile) - skip;
    *to = sink_tiles + k1 - first_tile - skip;
  }
  __device__ __forceinline__ bool part(int j, int tiles) const {  // some row of a tile that is worked on does not see all of it
    return (j < steps0 && !full(0, j)) || (tiles == 2 && j < steps1 && !full(1, j));
  }
};

// The page bits of a tile, spread over its 32 keys from column c on.
__device__ __forceinline__ uint32_t pages_of(uint32_t there, int c, int page_shift) {
  if (page_shift >= 7) return there ? 0xffffffffu : 0u;
  if (page_shift >= 5) return (there >> (c >> page_shift)) & 1 ? 0xffffffffu : 0u;
  uint32_t bits = 0;
  const int rows = 1 << page_shift;
  for (int q = 0; q < 32; q += rows)
    if ((there >> ((c + q) >> page_shift)) & 1) bits |= ((1u << rows) - 1u) << q;
  return bits;
}

template <int TQ>
__device__ __forceinline__ bool find_job(const TileArgs& g, int S, int rank, Job* job) {
  const approxifer_attention_args& a = g.a;
  // blocks of late queries see most: they come first
  int x = blockIdx.x / S;
  job->hk = x % a.Hkv;
  x /= a.Hkv;
  job->b = x % a.batch;
  const int block = g.blocks - 1 - x / a.batch;
  const int start = __ldg(a.q_start + job->b), queries = __ldg(a.q_start + job->b + 1) - start, held = __ldg(a.kv_len + job->b);
  const int skip = block * TQ * g.tokens;
  if (skip >= queries || start < 0 || (int64_t)start + queries > a.T) return false;
  job->tokens = g.tokens;
  job->token0 = start + skip;
  job->left = queries - skip;
  job->pos0 = held - queries + skip;
  job->window = a.window, job->sinks = a.sinks;
  const int last = job->pos0 + min(TQ * g.tokens, job->left) - 1;
  const int64_t room = a.table_pages << g.page_shift;
  job->p1 = last < room ? last : (int)(room - 1);
  job->lo = a.window && job->pos0 >= a.window ? job->pos0 - a.window + 1 : 0;
  const int seen_sinks = min(min(a.sinks, job->lo), job->p1 + 1);  // sinks before the window
  job->sink_tiles = seen_sinks > 0 ? (seen_sinks + kKeys - 1) / kKeys : 0;
  job->first_tile = max(job->lo / kKeys, job->sink_tiles);
  const int last_tile = job->p1 < 0 ? -1 : job->p1 / kKeys;
  job->steps = job->p1 < 0 ? 0 : job->sink_tiles + max(0, last_tile - job->first_tile + 1);
  const int last0 = job->last_pos(0);  // (of tile 0's rows)
  job->steps1 = TQ == 2 && job->tokens < job->left ? job->steps : 0;
  job->steps0 = job->steps1 == 0 ? job->steps : last0 < 0 ? 0 : min(job->steps, job->sink_tiles + max(0, last0 / kKeys - job->first_tile + 1));
  // a cluster's CTAs take consecutive parts of the steps; a query tile takes part in a first part of each as it does of all
  job->skip = (int)((int64_t)job->steps * rank / S);
  job->steps = (int)((int64_t)job->steps * (rank + 1) / S) - job->skip;
  job->steps0 = min(max(job->steps0 - job->skip, 0), job->steps);
  job->steps1 = min(max(job->steps1 - job->skip, 0), job->steps);
  return true;
}

__device__ __forceinline__ float max3(float a, float b, float c) {  // (a NaN is passed over; it makes its row NaN as a weight)
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// All ones over the elements of a pair of bfloat16 that are infinite or NaN.
__device__ __forceinline__ uint32_t bad_elements(uint32_t w) {
  const uint32_t e = (w & 0x7f807f80u) + 0x00800080u;  // an exponent of all ones carries into the sign's place
  return ((e >> 15) & 0x00010001u) * 0xffffu;
}

// S of a query tile and a key tile, both K-major in blocks of 64 columns.
template <int DP>
__device__ __forceinline__ void form_scores(uint32_t to, uint64_t q, uint64_t k) {
  constexpr int kBlock16 = kBlock >> 4;
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) mma_ss(to, q + (i / 4) * kBlock16 + 2 * (i % 4), k + (i / 4) * kBlock16 + 2 * (i % 4), mma_shape(kRows, kKeys), i > 0);
}

// Two warps meet (named barriers 1 .. 8); the second form says whether any of their threads wants something.
__device__ __forceinline__ void warps_meet(int id) { asm volatile("barrier.cta.sync.aligned %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool any_of_both(int id, bool want) {
  uint32_t any;
  asm volatile(
      "{\n.reg .pred p, q;\n"
      "setp.ne.u32 p, %2, 0;\n"
      "barrier.cta.red.or.pred.aligned q, %1, 64, p;\n"
      "selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(any)
      : "r"(id), "r"((uint32_t)want)
      : "memory");
  return any != 0;
}

// All softmax warps.
template <int TQ>
__device__ __forceinline__ void softmax_warps_meet() { asm volatile("barrier.cta.sync.aligned 15, %0;" ::"n"(TQ * 256) : "memory"); }

// The n-th (query tile, key tile) pair; the first or the last of its key tile.  (A query tile takes part from step 0 on.)
struct Item {
  int t, j;
  bool first, last;
};
template <int TQ>
__device__ __forceinline__ Item item_at(const Job& job, int n) {
  if (TQ == 1) return {0, n, true, true};
  const int both = min(job.steps0, job.steps1);
  if (n < 2 * both) return {n & 1, n >> 1, (n & 1) == 0, (n & 1) == 1};
  return {job.steps1 > 0 ? 1 : 0, n - both, true, true};
}

template <int DP, bool CLUSTER>
__global__ void __launch_bounds__(threads_of(DP), 3 - tiles_of(DP))
    attention_tile_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                          const __grid_constant__ TileArgs g) {
  constexpr int TQ = tiles_of(DP), kTile = tile_bytes(DP);
  constexpr int kScoreWarp = 8 * TQ, kOutWarp = kScoreWarp + 1, kCopyWarp = kScoreWarp + 2;
  // tensor memory: one tile S, P, O; two tiles S (with P over its first half) of each, O of each
  constexpr uint32_t kPCol = TQ == 1 ? kKeys : 0, kPStep = kKeys, kOutCol = TQ == 1 ? kKeys + kKeys / 2 : 2 * kKeys, kTmemCols = TQ * 256;
  extern __shared__ unsigned char raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(base);
  volatile int* abort = reinterpret_cast<volatile int*>(base + 512);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base + 516);
  volatile int* poison = reinterpret_cast<volatile int*>(base + 520);
  volatile uint32_t* pages_there = reinterpret_cast<volatile uint32_t*>(base + 576);  // [kMasks]: of tile j at j % kMasks, a bit per page
  const uint32_t full = smem_addr(bars), empty = full + 8 * kFulls, clean = empty + 8 * kStages, q_full = clean + 8 * kCleans, s_ready = q_full + 8,
                 s_free = s_ready + 16, p_ready = s_free + 8, pv_done = p_ready + 32;
  const uint32_t q_at = smem_addr(base + 1024), ring = q_at + TQ * kTile;
  auto landed = [&](int i) { return full + 8 * (i % kStages + (i & 1) * kStages); };
  auto landed_parity = [](int i) { return (uint32_t)(i / kStages >> 1) & 1; };  // (every second turn of a place is of the entry's kind)
  float* exchange = reinterpret_cast<float*>(base + 1024 + (TQ + kStages) * kTile);  // [tile][row]
  // (a cluster, at the end, over queries and ring) O of this CTA's part [tile][row][DP], maximum and sum [tile][row]
  float4* part_rows = reinterpret_cast<float4*>(base + 1024);
  float2* row_sums = reinterpret_cast<float2*>(base + 1024 + TQ * kRows * DP * 4);
  static_assert(TQ * kRows * (DP * 4 + 8) <= (TQ + kStages) * kTile, "a CTA's part exceeds queries and ring");
  const approxifer_attention_args& a = g.a;
  const int warp = warp_index(), lane = threadIdx.x % 32;
  unsigned int* count = &g_attention_tile_wait_timeouts;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kFulls; ++s) bar_init(full + 8 * s, 1);
    for (int s = 0; s < kStages; ++s) bar_init(empty + 8 * s, 1);
    for (int s = 0; s < kCleans; ++s) bar_init(clean + 8 * s, 1);
    bar_init(q_full, 1);
    bar_init(s_free, 8);
    for (int t = 0; t < TQ; ++t) bar_init(s_ready + 8 * t, 1), bar_init(p_ready + 16 * t, 4), bar_init(p_ready + 16 * t + 8, 4), bar_init(pv_done + 8 * t, 1);
    *abort = 0;
    *poison = 0;
    bar_init_done();
    prefetch_map(&q_map);
    prefetch_map(&k_map);
    prefetch_map(&v_map);
  }
  wait_for_inputs();
  Job job;
  const int S = CLUSTER ? (int)cluster_size() : 1, rank = CLUSTER ? (int)cluster_rank() : 0;
  if (!find_job<TQ>(g, S, rank, &job)) return;  // (all CTAs of a cluster or none)
  // (copies) the page of this lane's rows of a key tile, looked up a tile ahead
  const int32_t* table = a.block_table + (int64_t)job.b * a.table_stride;
  const int page_rows = 1 << g.page_shift, rows = min(page_rows, kKeys), per_tile = kKeys / rows;
  auto page_of = [&](int j) -> int32_t {
    if (j >= job.steps || lane >= per_tile) return -1;
    const int64_t at = (int64_t)((job.tile(j) * kKeys) >> g.page_shift) + lane;
    return at < a.table_pages ? __ldg(table + at) : -1;
  };
  int32_t page_ahead = warp == kCopyWarp ? page_of(0) : -1;
  if (warp == kScoreWarp) tmem_alloc(smem_addr(tmem_slot), kTmemCols);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  let_next_start();  // not before: the tensor memory is held

  // The softmax warps keep scores in registers; the four others give up theirs (two tiles: 512 x 104 + 128 x 64 = 640 x 96
  // registers at the launch; one: 256 x 96 + 128 x 48 = 384 x 80).
  if (warp < kScoreWarp) {
    if constexpr (TQ == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
    // ---- softmax and output: two threads to a row ----
    constexpr int kMine = kKeys / 2;  // keys, and kOut columns of the output, of a thread
    constexpr int kOut = DP / 2;
    const int t = warp / 8, half = warp / 4 % 2, quarter = warp % 4, r = quarter * 32 + lane;
    const int meet = 1 + t * 4 + quarter;  // the barrier of the two warps that share these rows
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_at = tmem + lanes + t * kKeys + half * kMine, p_at = tmem + lanes + kPCol + t * kPStep + half * (kMine / 2), o_at = tmem + lanes + kOutCol + t * DP + half * kOut;
    float* row_value = exchange + t * kRows + r;
    // the largest (or the sum) of what the row's two threads hold; both warps together
    auto of_both = [&](float v, auto combine) {
      if (half == 1) *row_value = v;
      warps_meet(meet);
      if (half == 0) *row_value = v = combine(v, *row_value);
      warps_meet(meet);
      if (half == 1) v = *row_value;
      return v;
    };
    const int in_tile = r / g.group, token = t * job.tokens + in_tile;
    const bool mine = in_tile < job.tokens && token < job.left;
    const int pos = job.pos0 + token;
    const bool flip = a.scale < 0.f;  // the running maximum is that of sign(scale) S
    // (of a zero scale just enough is left to keep what a row does not see at minus infinity)
    const float scale = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-37f);
    const uint64_t sc2 = pack2(scale, scale);
    const uint32_t all_pages = (1u << max(1, kKeys >> g.page_shift)) - 1u;
    int full_from, full_to;  // the steps in which every row of the tile sees every key
    job.full_steps(t, &full_from, &full_to);
    if (flip) full_to = 0;
    const int steps = job.steps_of(t);
    float m = mine ? -CUDART_INF_F : 0.f, l = 0.f;  // (rows that are not there never ask for another maximum)
    bool ok = true;
    int j = 0;
    for (; j < steps; ++j) {
      if (!(ok = warp_wait(s_ready + 8 * t, j & 1, abort, count))) break;
      tmem_fence_after();
      const uint32_t there = pages_there[j % kMasks];
      float s[kMine];
      tmem_ld32(s_at, *reinterpret_cast<uint32_t(*)[32]>(s));
      tmem_ld32(s_at + 32, *reinterpret_cast<uint32_t(*)[32]>(s + 32));
      tmem_wait_ld(*reinterpret_cast<uint32_t(*)[32]>(s));
      tmem_wait_ld(*reinterpret_cast<uint32_t(*)[32]>(s + 32));
      tmem_fence_before();
      if constexpr (TQ == 1) {
        __syncwarp();
        if (lane == 0) bar_arrive(s_free);
      }
      if (j < full_from || j >= full_to || there != all_pages) {  // what a row does not see becomes minus infinity
        if (flip) {
#pragma unroll
          for (int i = 0; i < kMine; ++i) s[i] = -s[i];
        }
#pragma unroll
        for (int c = 0; c < kMine; c += 32) {
          const int k = half * kMine + c;
          const uint32_t sees = job.sees(pos, job.tile(j) * kKeys + k) & pages_of(there, k, g.page_shift);
          if (__any_sync(0xffffffffu, sees != 0xffffffffu)) {
#pragma unroll
            for (int i = 0; i < 32; ++i) s[c + i] = sees & (1u << i) ? s[c + i] : -CUDART_INF_F;
          }
        }
      }
      float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
      for (int i = 0; i < kMine; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) top[k] = max3(top[k], s[i + 2 * k], s[i + 2 * k + 1]);
      top[0] = fmaxf(max3(top[0], top[1], top[2]), top[3]);
      // the last P has been used, O is whole (two tiles: so S says already, which follows them on the tensor cores)
      if (TQ == 1 && j > 0 && !(ok = warp_wait(pv_done, (j - 1) & 1, abort, count))) break;
      tmem_fence_after();
      // (the vote also keeps P from being written before both warps have read the scores that it may lie over)
      if (any_of_both(meet, mine && (m == -CUDART_INF_F || (top[0] - m) * scale > kGrowth))) {
        const float most = of_both(top[0], [](float x, float y) { return fmaxf(x, y); });
        const bool grow = mine && m != -CUDART_INF_F && (most - m) * scale > kGrowth;
        const float keep = grow ? pow2((m - most) * scale) : 1.f;
        if (mine && (grow || m == -CUDART_INF_F)) m = most;  // (at minus infinity nothing is summed yet but zeros)
        l *= keep;
        if (j > 0 && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
          for (int c = 0; c < kOut; c += 16) {
            uint32_t v[16];
            tmem_ld16(o_at + c, v);
            tmem_wait_ld(v);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * keep);
            tmem_st16(o_at + c, v);
          }
          tmem_wait_st();
          tmem_fence_before();
        }
        warps_meet(meet);  // O is whole again before either warp hands over its weights
        tmem_fence_after();
      }
      const float shift_by = m == -CUDART_INF_F ? 0.f : -m * scale;
      const uint64_t sh2 = pack2(shift_by, shift_by);
      uint64_t sum2[2] = {0, 0};
#pragma unroll
      for (int c = 0; c < kMine; c += 32) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          float x, y;
          unpack2(fma2(pack2(s[c + i], s[c + i + 1]), sc2, sh2), x, y);
          x = pow2(x), y = pow2(y);
          sum2[(i / 2) & 1] = add2(sum2[(i / 2) & 1], pack2(x, y));
          p[i / 2] = pack_bf16x2(x, y);
        }
        tmem_st16(p_at + c / 2, p);
      }
      tmem_wait_st();
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(p_ready + 16 * t + 8 * half);
      float u, v;
      unpack2(add2(sum2[0], sum2[1]), u, v);
      l += u + v;
    }
    // After a wait that gave up the warp keeps the meetings of the steps that it leaves out: the other warp of its rows may be on
    // its way to them, and they have no limit of their own.
    for (; j < steps; ++j)
      if (any_of_both(meet, false)) warps_meet(meet), warps_meet(meet), warps_meet(meet);
    if (steps > 0) {
      l = of_both(l, [](float x, float y) { return x + y; });
      if (ok) ok = warp_wait(pv_done + 8 * t, TQ == 1 ? (steps - 1) & 1 : 0, abort, count);
      tmem_fence_after();
    }
    if constexpr (CLUSTER) softmax_warps_meet<TQ>();  // no product reads shared memory any more, of either tile
    if (ok) {
      // One CTA: O / sum, by way of the tile's queries' place in shared memory (a warp keeps to its own rows and columns) into
      // whole rows.  A cluster: O as it is into shared memory, with the row's maximum and sum.
      const float inv = CLUSTER ? 1.f : l == 0.f ? 0.f : 1.f / l;
      const bool add_back = *poison != 0;
      unsigned char* own_rows = base + 1024 + t * kTile + (half * 4 + quarter) * 32 * kOut * 2;
      constexpr int kCols = kOut / 8;  // 16-byte columns
      if (CLUSTER && half == 0) row_sums[t * kRows + r] = make_float2(m, l);
#pragma unroll 1
      for (int c = 0; c < kOut; c += 16) {
        float y[16];
        if (steps > 0) {
          uint32_t v[16];
          tmem_ld16(o_at + c, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = l == 0.f ? 0.f : __uint_as_float(v[i]) * inv;
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = 0.f;
        }
        if (mine && add_back) {
          // infinities and NaN that were taken out of tiles seen in part, for the rows that do see them
          const int d0 = half * kOut + c;
#pragma unroll 1
          for (int j = 0; j < job.steps; ++j) {
            if (!job.part(j, TQ)) continue;
            const int k0 = job.tile(j) * kKeys;
#pragma unroll 1
            for (int k = k0; k < k0 + kKeys && k <= min(pos, job.p1); ++k) {
              if (a.window && k <= pos - a.window && k >= a.sinks) continue;
              const int32_t page = __ldg(table + (k >> g.page_shift));
              if (page < 0 || page >= a.num_pages) continue;
              const bf16* v = reinterpret_cast<const bf16*>(a.v_cache) + page * a.vc_pstride + job.hk * a.vc_hstride +
                              (k & ((1 << g.page_shift) - 1)) * a.vc_rstride;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float x = d0 + i < a.D ? widen(v[d0 + i]) : 0.f;
                if (!isfinite(x)) y[i] += x;
              }
            }
          }
        }
        if constexpr (CLUSTER) {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            part_rows[(t * kRows + r) * (DP / 4) + (((half * kOut + c + i) / 4) ^ (r & 7))] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; i += 8)
            *reinterpret_cast<uint4*>(own_rows + lane * kOut * 2 + ((((c + i) / 8) ^ (lane & (kCols - 1))) << 4)) =
                make_uint4(pack_bf16x2(y[i], y[i + 1]), pack_bf16x2(y[i + 2], y[i + 3]), pack_bf16x2(y[i + 4], y[i + 5]), pack_bf16x2(y[i + 6], y[i + 7]));
        }
        __syncwarp();
      }
      const int64_t to = mine ? (int64_t)(job.token0 + token) * a.o_tstride + (int64_t)(job.hk * g.group + r % g.group) * a.o_hstride : -1;
#pragma unroll 4
      for (int x = lane; !CLUSTER && x < 32 * kCols; x += 32) {
        const int row = x / kCols, col = x % kCols, d = half * kOut + col * 8;
        const int64_t at = __shfl_sync(0xffffffffu, to, row);
        if (at >= 0 && d < a.D)
          *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(a.out) + at + d) = *reinterpret_cast<const uint4*>(own_rows + row * kOut * 2 + ((col ^ (row & (kCols - 1))) << 4));
      }
    }
    tmem_fence_before();
  } else {
    if constexpr (TQ == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == kCopyWarp) {
      // ---- copies ----
      // The queries of the tiles that have a step, and of no other: the first product is what waits for them.  A copy that nothing
      // waits for would land in rows that the output is staged in meanwhile, or in the memory of the SM's next CTA.
      if (lane == 0 && job.steps > 0) {
        bar_expect(q_full, ((job.steps0 > 0) + (job.steps1 > 0)) * (DP / 64) * g.group * job.tokens * 128);
        for (int t = 0; t < TQ; ++t)
          for (int c = 0; c < DP / 64 && job.steps_of(t) > 0; ++c)
            tma_3d(q_at + t * kTile + c * kBlock, &q_map, c * 64, job.hk * g.group, job.token0 + t * job.tokens, q_full);
      }
      bool ok = true;
      for (int j = 0; j < job.steps && ok; ++j) {
        const int k0 = job.tile(j) * kKeys;
        int32_t page = page_ahead;
        page_ahead = page_of(j + 1);
        const bool there = page >= 0 && page < a.num_pages;
        if (!there) page = (int32_t)a.num_pages;  // beyond the array: zeros
        const uint32_t mask = __ballot_sync(0xffffffffu, there);
        const int row = k0 & (page_rows - 1);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int i = 2 * j + v, s = i % kStages, turn = i / kStages;
          if (turn > 0 && !(ok = warp_wait(empty + 8 * s, (turn - 1) & 1, abort, count))) break;
          if (lane == 0) {
            if (v == 0) pages_there[j % kMasks] = mask;
            bar_expect(landed(i), kTile);
          }
          __syncwarp();
          if (lane < per_tile)
            for (int c = 0; c < DP / 64; ++c)
              tma_4d(ring + s * kTile + c * kBlock + lane * rows * 128, v ? &v_map : &k_map, c * 64, row, job.hk, page, landed(i));
        }
      }
    } else if (warp == kScoreWarp) {
      // ---- S (one tile) ----
      if (TQ == 1 && job.steps > 0 && warp_wait(q_full, 0, abort, count)) {
        for (int j = 0; j < job.steps; ++j) {
          const int i = 2 * j, stage = i % kStages;
          const uint64_t ks = desc_k_major(ring + stage * kTile);
          if (!warp_wait(landed(i), landed_parity(i), abort, count)) break;
          if (j > 0 && !warp_wait(s_free, (j - 1) & 1, abort, count)) break;  // the last S is in registers
          tmem_fence_after();
          if (elect_one()) {
            form_scores<DP>(tmem, desc_k_major(q_at), ks);
            mma_commit(s_ready);
            mma_commit(empty + 8 * stage);
          }
          __syncwarp();
        }
      }
    } else if (warp == kOutWarp) {
      // ---- O (one tile); S and O (two) ----
      // Items: (query tile, key tile) pairs in the order of the key tiles, both query tiles of a key tile while both take part,
      // then those of tile 1.  Every key tile has an item; its values are given back with the last, its keys with its last S.
      const int items = job.steps0 + job.steps1;
      bool ok = items > 0;
      int keys_in = 1;
      if (TQ == 2 && ok) {
        ok = warp_wait(q_full, 0, abort, count) && warp_wait(landed(0), landed_parity(0), abort, count);
        if (ok && elect_one()) {
#pragma unroll
          for (int t = 0; t < TQ; ++t)
            if (job.steps_of(t) > 0) {
              form_scores<DP>(tmem + t * kKeys, desc_k_major(q_at + t * kTile), desc_k_major(ring));
              mma_commit(s_ready + 8 * t);
            }
          mma_commit(empty);
        }
        __syncwarp();
      }
      for (int n = 0; n < items && ok; ++n) {
        const Item x = item_at<TQ>(job, n);
        const int value = 2 * x.j + 1, stage = value % kStages, next_key = (value + 1) % kStages;
        const bool more = x.j + 1 < job.steps_of(x.t);
        if (x.first && !(ok = warp_wait(clean + 8 * (x.j % kCleans), (x.j / kCleans) & 1, abort, count))) break;  // landed, and looked through
        if (TQ == 2 && more && keys_in == x.j + 1) {
          if (!(ok = warp_wait(landed(value + 1), landed_parity(value + 1), abort, count))) break;
          ++keys_in;
        }
        const uint64_t vs = desc_mn_major(ring + stage * kTile, kBlock);
        const uint32_t to = tmem + kOutCol + x.t * DP, from = tmem + kPCol + x.t * kPStep;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(ok = warp_wait(p_ready + 16 * x.t + 8 * half, x.j & 1, abort, count))) break;
          tmem_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kKeys / 32; ++k)
              mma_ts(to, from + (half * (kKeys / 32) + k) * 8, vs + (half * (kKeys / 32) + k) * 128, mma_shape(kRows, DP, true), x.j > 0 || half > 0 || k > 0);
            if (half == 1) {
              if (TQ == 1 || !more) mma_commit(pv_done + 8 * x.t);
              if (x.last) mma_commit(empty + 8 * stage);
              if (TQ == 2 && more) {  // over the P that has just been used
                form_scores<DP>(tmem + x.t * kKeys, desc_k_major(q_at + x.t * kTile), desc_k_major(ring + next_key * kTile));
                mma_commit(s_ready + 8 * x.t);
                if (x.t == 1 || x.j + 1 >= job.steps1) mma_commit(empty + 8 * next_key);
              }
            }
          }
          __syncwarp();
        }
      }
    } else {
      // ---- values of tiles that are seen in part ----
      bool ok = true;
      for (int j = 0; j < job.steps && ok; ++j) {
        const int i = 2 * j + 1, s = i % kStages;
        if (!(ok = warp_wait(landed(i), landed_parity(i), abort, count))) break;
        const bool part = job.part(j, TQ);
        if (part) {
          uint4* v = reinterpret_cast<uint4*>(base + 1024 + (TQ + s) * kTile);
          const int k0 = job.tile(j) * kKeys;
#pragma unroll 1
          for (int x0 = lane; x0 < kTile / 16; x0 += 32 * 4) {
            uint4 u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = v[x0 + 32 * e];
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) any |= bad_elements(u[e].x) | bad_elements(u[e].y) | bad_elements(u[e].z) | bad_elements(u[e].w);
            if (any == 0) continue;
#pragma unroll 1
            for (int x = x0; x < x0 + 32 * 4; x += 32) {
              uint4 w = v[x];
              const uint32_t b0 = bad_elements(w.x), b1 = bad_elements(w.y), b2 = bad_elements(w.z), b3 = bad_elements(w.w);
              if ((b0 | b1 | b2 | b3) == 0) continue;
              w.x &= ~b0, w.y &= ~b1, w.z &= ~b2, w.w &= ~b3;
              v[x] = w;
              const int at = k0 + (x / 8) % kKeys;
              if (at <= job.p1 && (at >= job.lo || at < job.sinks)) *poison = 1;  // (a row of this CTA may see it)
            }
          }
          async_proxy_fence();
        }
        __syncwarp();
        if (lane == 0) bar_arrive(clean + 8 * (j % kCleans));
      }
    }
  }
  __syncwarp();
  __syncthreads();
  drain_if_aborted(abort);
  if (warp == kScoreWarp) {
    tmem_fence_after();
    tmem_free(tmem, kTmemCols);
  }
  if constexpr (CLUSTER) {
    // The CTAs' parts of every row, in order: each CTA joins its share of the rows, a warp to a row.
    cluster_sync();
    if (warp < kScoreWarp) {
      const float scale = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-37f);
      const uint32_t parts = smem_addr(part_rows), sums = smem_addr(row_sums);
      for (int x = TQ * kRows * rank / S + warp; x < TQ * kRows * (rank + 1) / S; x += kScoreWarp) {
        const int t = x / kRows, r = x % kRows, token = t * job.tokens + r / g.group;
        if (r / g.group >= job.tokens || token >= job.left) continue;
        float2 ml[kMaxSplit];
        float best = -CUDART_INF_F;
#pragma unroll
        for (int s = 0; s < kMaxSplit; ++s) {
          ml[s] = s < S ? peer_load2(peer_smem(sums + x * 8, s)) : make_float2(-CUDART_INF_F, 0.f);
          best = fmaxf(best, ml[s].x);
        }
        if (best == -CUDART_INF_F) best = 0.f;
        const int c = lane * (DP / 32);  // this lane's columns
        const uint32_t at = parts + (x * (DP / 4) + ((c / 4) ^ (r & 7))) * 16 + (c % 4) * 4;
        float total = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kMaxSplit; ++s) {
          if (s >= S) continue;
          const float k = pow2((ml[s].x - best) * scale);
          total = fmaf(k, ml[s].y, total);
          if constexpr (DP == 128) {
            const float4 v = peer_load(peer_smem(at, s));
            y[0] = fmaf(k, v.x, y[0]), y[1] = fmaf(k, v.y, y[1]), y[2] = fmaf(k, v.z, y[2]), y[3] = fmaf(k, v.w, y[3]);
          } else {
            const float2 v = peer_load2(peer_smem(at, s));
            y[0] = fmaf(k, v.x, y[0]), y[1] = fmaf(k, v.y, y[1]);
          }
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        bf16* out = reinterpret_cast<bf16*>(a.out) + (int64_t)(job.token0 + token) * a.o_tstride + (int64_t)(job.hk * g.group + r % g.group) * a.o_hstride + c;
        if (c < a.D) {
          if constexpr (DP == 128) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
          else *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(y[0] * inv, y[1] * inv);
        }
      }
    }
    cluster_sync();  // (a CTA's shared memory stays until all have read it)
  }
}

template <int DP, bool CLUSTER>
cudaError_t launch_split(const TileArgs& g, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const DeviceInfo& dev, int64_t ctas, int split,
                         cudaStream_t stream) {
  auto kernel = attention_tile_kernel<DP, CLUSTER>;
  struct Tag {};
  const cudaError_t e = ensure_dynamic_smem<Tag>(kernel, dev.ordinal, smem_bytes(DP));
  if (e != cudaSuccess) return e;
  return launch_kernel(kernel, ctas * split, threads_of(DP), smem_bytes(DP), split, stream, q, k, v, g);
}

template <int DP>
cudaError_t launch_one(const TileArgs& g, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, cudaStream_t stream) {
  const DeviceInfo* dev;
  const cudaError_t e = current_device_info(&dev);
  if (e != cudaSuccess) return e;
  const approxifer_attention_args& a = g.a;
  const int64_t ctas = (int64_t)g.blocks * a.batch * a.Hkv;
  // Few query blocks: as many CTAs to each, along the keys, as the GPU holds, each with three tiles of keys or more.  (The
  // lengths are on the device: what a block can see at most says how far it is worth cutting.)  Measured, one CTA a block
  // against the cluster, us: 2 queries at 4,000 keys, 1 key head of 128: 62 / 16; 10 at 4,000, 8 heads of 64: 44 / 13; 64 at
  // 2,048, 2 heads of 128: 38 / 22; 80 blocks of 64 cut in two for two CTAs on every SM: 31 / 35, hence one CTA to an SM.
  int64_t most = a.table_pages * a.page_size;
  if (a.window && (int64_t)a.window + a.max_q + a.sinks < most) most = (int64_t)a.window + a.max_q + a.sinks;
  const int held = dev->sms * 3 / 4;
  int split = 1;
  while (split < kMaxSplit && ctas * split * 2 <= held && most >= (int64_t)split * 2 * 3 * kKeys) split *= 2;
  return split > 1 ? launch_split<DP, true>(g, q, k, v, *dev, ctas, split, stream) : launch_split<DP, false>(g, q, k, v, *dev, ctas, 1, stream);
}

}  // namespace

cudaError_t read_attention_tile_wait_timeouts(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_attention_tile_wait_timeouts, sizeof(*out)); }
cudaError_t reset_attention_tile_wait_timeouts() {
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_attention_tile_wait_timeouts, &zero, sizeof(zero));
}

bool attention_tile_eligible(const approxifer_attention_args& a) {
  const int64_t limit = 1LL << 38;
  return a.D % 8 == 0 && a.D <= 128 && a.Hq / a.Hkv <= kRows && a.num_pages >= 1 && a.page_size >= 8 && exact_log2(a.page_size) > 0 &&
         a.table_pages * a.page_size < (1LL << 30) && aligned16(a.q) && aligned16(a.k_cache) && aligned16(a.v_cache) && aligned16(a.out) &&
         (a.q_tstride | a.q_hstride | a.o_tstride | a.o_hstride | a.kc_pstride | a.kc_hstride | a.kc_rstride | a.vc_pstride | a.vc_hstride | a.vc_rstride) % 8 == 0 &&
         a.q_tstride > 0 /* (a tensor map's strides; one query for all tokens is the element-wise kernel's) */ && a.q_tstride < limit && a.q_hstride < limit && a.kc_pstride < limit && a.kc_hstride < limit && a.kc_rstride < limit && a.vc_pstride < limit &&
         a.vc_hstride < limit && a.vc_rstride < limit && a.sinks < (1 << 30) && a.window < (1 << 30);
}

cudaError_t launch_attention_tile(const approxifer_attention_args& a, cudaStream_t stream) {
  TileArgs g{};
  g.a = a;
  if (g.a.max_q > a.T) g.a.max_q = (int32_t)a.T;  // (no sequence has more queries than the call: a loose bound launches no CTAs for nothing)
  g.group = a.Hq / a.Hkv;
  g.tokens = kRows / g.group;
  const int per_cta = tiles_of(a.D <= 64 ? 64 : 128) * g.tokens;
  g.blocks = (int)(((int64_t)g.a.max_q + per_cta - 1) / per_cta);
  g.page_shift = exact_log2(a.page_size);
  const int dp = a.D <= 64 ? 64 : 128;
  CUtensorMap q, k, v;
  const uint64_t qe[3] = {(uint64_t)a.D, (uint64_t)a.Hq, (uint64_t)a.T}, qs[3] = {1, (uint64_t)a.q_hstride, (uint64_t)a.q_tstride};
  const uint32_t qb[3] = {64, (uint32_t)g.group, (uint32_t)g.tokens};
  const uint64_t ce[4] = {(uint64_t)a.D, (uint64_t)a.page_size, (uint64_t)a.Hkv, (uint64_t)a.num_pages};
  const uint64_t kst[4] = {1, (uint64_t)a.kc_rstride, (uint64_t)a.kc_hstride, (uint64_t)a.kc_pstride};
  const uint64_t vst[4] = {1, (uint64_t)a.vc_rstride, (uint64_t)a.vc_hstride, (uint64_t)a.vc_pstride};
  const uint32_t cb[4] = {64, (uint32_t)(a.page_size < kKeys ? a.page_size : kKeys), 1, 1};
  cudaError_t e;
  if ((e = make_tensor_map(&q, a.q, 3, qe, qs, qb)) != cudaSuccess || (e = make_tensor_map(&k, a.k_cache, 4, ce, kst, cb)) != cudaSuccess ||
      (e = make_tensor_map(&v, a.v_cache, 4, ce, vst, cb)) != cudaSuccess)
    return e;
  return dp == 64 ? launch_one<64>(g, q, k, v, stream) : launch_one<128>(g, q, k, v, stream);
}

}  // namespace approxifer
