// Attention of one new token per sequence over the full cache, every sequence of its own length.
//
// A row (sequence, KV head) is cut into blocks of 16 KB of K and V (bf16, 128 dims: 32 tokens), a wave's work at a time.  (Blocks of twice that at 128 dims: one
// sequence of 512K tokens 325 us instead of 318, and short rows end in larger remainders.)  All rows, one after the other, are divided
// over the launch's waves, whatever their lengths: a row weighs its blocks and kRowWeight more for its beginning and end, and every wave gets the same
// weight, a run of blocks that may hold several rows and two parts of rows at most, one that continues a row and one that begins
// one.  A wave finds its share from the lengths alone, which it reads on the device (64 of them at a time, summed over the wave), and goes through it without waiting for
// any other: its loads run a block ahead of its arithmetic, into the next row too.  A whole row goes straight to `out`; parts stay in LDS until the
// four waves of the workgroup, whose shares are neighbours, are done, and are merged there, (max, sum, accumulator) by (max, sum, accumulator).  What the
// workgroup then has not got the whole of goes to scratch, one row that it continues and one that it begins at most, and join_kernel merges that.
// (With shares for workgroups, whose four waves took a row's blocks in turn and merged them at its end, a row cost as much as 8 blocks, and 64 sequences of
// 1 to 32K tokens 88 us instead of 80.)
//
// One workgroup per CU.  (With two, the older one of a CU and some XCDs get ahead: one sequence of 512K tokens ends its loop between 267 and 321 us, with one between 294
// and 308.)  Bound by HBM: K and V are read once for 16 heads of a group at a time (fp32: 8).  Short calls are bound by latency: lengths, pages, the first block and the
// join come one after the other, 6.5 us of a call, and a block takes a wave 1.35 us (fp32 1.8) however little the others read.
#include "device_utils.h"
#include "full_cache.h"

namespace sagekv {

namespace {

constexpr int NW = 4;  // waves of a workgroup

// ---- rows, weights and shares ------------------------------------------------------------------
// Lengths do not change while a launch runs (if they do, results are wrong, but no access leaves its buffer): through the constant address space they come
// by scalar loads, which nothing else waits for.  (A vector load of a length in the middle of a share waits for all of K and V that is in flight.)
__device__ __forceinline__ int length_of(const CacheAttnParams& p, int prob) {
  return ((const __attribute__((address_space(4))) int*)p.lens)[prob];
}

// The blocks of a row of len tokens that hold attended tokens.  With a window those of the first S and of the last W tokens.
template <int BT>
struct RowBlocks {
  int len, n;      // tokens; blocks
  int head, skip;  // blocks from `head` on lie `skip` blocks further
  __device__ __forceinline__ int token(int block) const { return (block < head ? block : block + skip) * BT; }
  __device__ __forceinline__ RowBlocks() {}
  __device__ __forceinline__ RowBlocks(const CacheAttnParams& p, int length) {
    len = length < 0 ? 0 : length < p.max_len ? length : p.max_len;
    n = (len + BT - 1) / BT;
    head = n;
    skip = 0;
    if (p.W > 0) {
      const int sinks = (p.S + BT - 1) / BT, tail = (len - p.W) / BT;  // blocks of the sink tokens, first block of the window
      if (len > p.W && tail > sinks) {
        head = sinks;
        skip = tail - sinks;
        n -= skip;
      }
    }
  }
};
// The shares: `more` of them of size + 1, the others of size.
struct Shares {
  int n, size, more;
  __device__ __forceinline__ Shares(int total, int n_) : n(n_), size(total / n_), more(total - total / n_ * n_) {}
  __device__ __forceinline__ int begin(int i) const { return i * size + min(i, more); }
  __device__ __forceinline__ int of(int at) const {
    const int large = more * (size + 1);
    return at < large ? at / (size + 1) : more + (at - large) / size;
  }
};

// What n problems have: blocks, problems with tokens, the most blocks (of one row of each problem); and the last one's length.
struct Census {
  int blocks, rows, most, length;
  template <int BT>
  __device__ __forceinline__ void take(const CacheAttnParams& p, int first, int n) {
    blocks = rows = most = length = 0;
    for (int i0 = 0; i0 < n; i0 += 4) {
      int len[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) len[i] = p.lens[first + min(i0 + i, n - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = i0 + i < n ? RowBlocks<BT>(p, len[i]).n : 0;
        blocks += b;
        rows += b > 0;
        most = max(most, b);
      }
      length = len[3];
    }
  }
};

// A wave's share, part by part.
template <int BT>
struct Walk {
  int at, end;        // what is left of it, in weights
  int cuts;           // > 0: every row weighs that much, and each unit of its weight is an equal part of it
  int prob, c, done;  // the row that `at` is in, and what of its weight lies before
  RowBlocks<BT> row;
  __device__ __forceinline__ int weight() const { return row.n == 0 ? 0 : cuts ? cuts : row.n + kRowWeight; }
  // wave: its number in the launch
  __device__ __forceinline__ Shares start(const CacheAttnParams& p, int wave, int lane) {
    int lo = 0, n = p.P, before = 0;
    Shares shares(0, 1);
    bool counted = false;
    at = end = 0;
    for (;;) {  // a problem out of 64, of 64 * 64, ...
      const int per = (n + 63) / 64, first = lane * per, mine = max(0, min(per, n - first));
      Census census;
      census.take<BT>(p, lo + first, mine);
      const int blocks = wave_scan_incl(census.blocks) * p.Hkv, rows = wave_scan_incl(census.rows) * p.Hkv;
      if (!counted) {
        counted = true;
        const int all_blocks = __builtin_amdgcn_readlane(blocks, 63), all_rows = __builtin_amdgcn_readlane(rows, 63);
        // Whole rows, a workgroup's, two waves' or a wave's each, where the longest one takes hardly longer than an even share of all blocks does: parts of rows
        // to be joined cost about four rounds.  (256 rows of 7 heads x 128 dims, us, split and whole: 260 tokens 20.5 14.0, 512 26.5 16.8, 768 31.7 22.1; 8 rows of
        // 4 heads: 260 12.3 12.0, 384 12.1 12.0, 512 12.0 14.0, 768 12.0 17.9.)
        const RowCuts whole(all_rows);
        cuts = whole.rounds(wave_max_i(census.most)) <= all_blocks / kAttnWaves + kWholeRounds ? whole.cuts : 0;
        const int total = cuts ? all_rows * cuts : all_blocks + all_rows * kRowWeight, busy = min(total, p.n_waves);
        shares = Shares(total, max(1, busy));
        if (wave >= busy) return shares;
        at = shares.begin(wave);
        end = shares.begin(wave + 1);
      }
      // the first lane whose problems reach beyond the share's begin
      const int incl = cuts ? rows * cuts : blocks + rows * kRowWeight;
      const int hit = max(__ffsll((unsigned long long)__ballot(before + incl > at)) - 1, 0);
      before += hit > 0 ? __builtin_amdgcn_readlane(incl, hit - 1) : 0;
      lo += hit * per;
      n = min(per, n - hit * per);
      if (per > 1) continue;
      row = RowBlocks<BT>(p, __builtin_amdgcn_readlane(census.length, hit));
      break;
    }
    prob = lo;
    const int w = max(weight(), 1), in_problem = at - before;
    c = min(in_problem / w, p.Hkv - 1);
    done = in_problem - c * w;
    return shares;
  }
  int block0, block1;  // the part of that row: its blocks
  int row_end;         // where the row ends, in weights
  // the next part that holds blocks; false: none is left
  __device__ __forceinline__ bool next(const CacheAttnParams& p) {
    while (at < end) {
      const int w = weight();
      if (done >= w) {
        done = 0;
        if (++c == p.Hkv) {
          c = 0;
          do {
            if (++prob == p.P) return false;
            row = RowBlocks<BT>(p, length_of(p, prob));
          } while (row.n == 0);
        }
        continue;
      }
      const int take = min(w - done, end - at);
      row_end = at - done + w;
      if (cuts) {  // 1, 2 or 4
        block0 = row.n * done / cuts;
        block1 = row.n * (done + take) / cuts;
      } else {
        block0 = max(done - kRowWeight, 0);
        block1 = max(done + take - kRowWeight, 0);
      }
      at += take;
      done += take;
      if (block1 > block0) return true;
    }
    return false;
  }
};

// Problems without tokens: out = 0, lse = -infinity.  length: of the workgroup's first problem, read early.
__device__ __forceinline__ void clear_empty(const CacheAttnParams& p, int length) {
  for (int prob = blockIdx.x; prob < p.P;) {
    if (length <= 0) {
      for (int i = threadIdx.x; i < p.Hq * p.D; i += blockDim.x) p.out[(int64_t)prob * p.Hq * p.D + i] = 0.f;
      if (p.lse)
        for (int i = threadIdx.x; i < p.Hq; i += blockDim.x) p.lse[(int64_t)prob * p.Hq + i] = -INFINITY;
      if (p.by_row)
        for (int c = threadIdx.x; c < p.Hkv; c += blockDim.x) p.joins[prob * p.Hkv + c].first = -1;
    }
    prob += gridDim.x;
    if (prob < p.P) length = length_of(p, prob);
  }
}

// Tokens of a row that are attended; a block of n tokens from t0 on: are there any that are not?
struct Mask {
  int len, S, tail;  // tokens t < S or t >= tail, and t < len
  __device__ __forceinline__ Mask(const CacheAttnParams& p, int len_) : len(len_), S(p.S), tail(p.W > 0 ? len_ - p.W : 0) {}
  __device__ __forceinline__ bool at(int t) const { return t < len && (t < S || t >= tail); }
  __device__ __forceinline__ bool cuts(int t0, int n) const { return t0 + n > len || (tail > t0 && t0 + n > S); }
};

typedef const __attribute__((address_space(1))) char* GlobalBytes;  // (of a plain pointer made from two integers the compiler knows no address space)

// The block that a wave loads next.
template <int BT>
struct Ahead : Walk<BT> {
  static constexpr int GPB = BT / 16;  // groups of 16 tokens of a block
  int it;      // block `it` of the part
  uint64_t key_at, value_at;  // of the next 64 groups, one per lane: where their tokens begin, in K and in V
  bool valid;  // there is a block
  __device__ __forceinline__ int token0() const { return this->row.token(this->block0 + it); }
  __device__ __forceinline__ void step(const CacheAttnParams& p, int lane) {
    if (this->block0 + ++it >= this->block1) {
      valid = this->next(p);
      if (!valid) return;
      it = 0;
    }
    if ((it * GPB & 63) != 0) return;
    const int block = min(this->block0 + it + lane / GPB, this->block1 - 1);
    const int t = min(this->row.token(block) + lane % GPB * 16, this->row.len - 1), in = t & (int)((1u << p.cache.shift) - 1u);
    int page = this->prob;  // a dense cache's "page" is the problem
    if (p.cache.table) {
      page = p.cache.table[(int64_t)this->prob * p.cache.pitch + (t >> p.cache.shift)];
      page = page < 0 ? 0 : page >= p.cache.n_blocks ? p.cache.n_blocks - 1 : page;
    }
    key_at = (uint64_t)(p.cache.K + this->c * p.cache.ks_head + page * p.cache.ks_block + (int64_t)in * p.cache.ks_token);
    value_at = (uint64_t)(p.cache.V + this->c * p.cache.vs_head + page * p.cache.vs_block + (int64_t)in * p.cache.vs_token);
  }
  // Group g of the block's groups of 16 tokens, in K or V: where its tokens begin, and how many of them lie behind the first (those behind the row are
  // read as its last one).
  struct Group {
    GlobalBytes at;
    int last;
  };
  __device__ __forceinline__ Group group(uint64_t at, int g) const {
    const int k = (it * GPB + g) & 63;
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)at, k), hi = __builtin_amdgcn_readlane((uint32_t)(at >> 32), k);
    return {(GlobalBytes)((uint64_t)hi << 32 | lo), max(this->row.len - 1 - token0() - 16 * g, 0)};
  }
  __device__ __forceinline__ Group keys(int g) const { return group(key_at, g); }
  __device__ __forceinline__ Group values(int g) const { return group(value_at, g); }
};
// 16 bytes at `offset` of the group's token t of this lane: a wave-uniform address and 32 bits per lane (a token's stride has less than 24).
template <bool STREAM, typename Group>
__device__ __forceinline__ uint4 load_token(const Group& g, int s_token, int t, int offset) {
  const auto* at = (const __attribute__((address_space(1))) u32x4_t*)(g.at + (uint32_t)(__umul24((unsigned)min(t, g.last), (unsigned)s_token) + (unsigned)offset));
  const u32x4_t v = STREAM ? __builtin_nontemporal_load(at) : *at;
  return make_uint4(v.x, v.y, v.z, v.w);
}

// ---- what becomes of a part ----------------------------------------------------------------------
// In LDS a part is its accumulators [heads][D] and (max, sum) per head, not normalised.
__device__ __forceinline__ int64_t part_at(const CacheAttnParams& p, int group, bool begins) { return ((int64_t)group * 2 + begins) * p.G; }

// A part that a wave leaves in LDS: the first one of its share, or its last one.  row < 0: there is none.
struct Part {
  int row, block0, block1, n, row_end;  // of a row of n blocks
  __device__ __forceinline__ bool whole() const { return block0 == 0 && block1 == n; }
};

// The group's heads that a workgroup handles; the first ones' workgroups see to what there is once per row.
struct Heads {
  int first, n;
  __device__ __forceinline__ explicit Heads(const CacheAttnParams& p) : first(blockIdx.y * p.heads), n(min(p.heads, p.G - first)) {}
};

// A row that a wave has for itself.
template <int D>
__device__ __forceinline__ void write_row(const CacheAttnParams& p, Heads heads, int row, int lane, const float* acc, const float2* ml) {
  const int64_t head0 = (int64_t)row * p.G + heads.first;
  for (int i = lane; i < heads.n * (D / 4); i += 64) {
    const float l = ml[i / (D / 4)].y, f = l == 0.f ? 0.f : 1.f / l;
    const float4 a = reinterpret_cast<const float4*>(acc)[i];
    reinterpret_cast<float4*>(p.out + head0 * D)[i] = l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(a.x * f, a.y * f, a.z * f, a.w * f);
  }
  if (p.lse && lane < heads.n) p.lse[head0 + lane] = ml[lane].y == 0.f ? -INFINITY : fmaf(ml[lane].x, p.join_scale, logf(ml[lane].y));
  if (p.by_row && heads.first == 0 && lane == 0) p.joins[row].first = -1;
}

// The end of a workgroup, behind a barrier: its waves' parts, in order, those of a row merged.  Part 2 w is the first one of wave w, 2 w + 1 its last
// one; part k has its accumulators at acc + k * stride.
template <int D, int HEADS>
__device__ __forceinline__ void finish_group(const CacheAttnParams& p, Heads heads, const Shares& shares, const Part (&left)[2 * NW], const float* acc,
                                             int stride, const float2 (&ml)[2 * NW][HEADS]) {
  const int group = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const float cexp = p.join_scale * 1.44269502162933349609375f;
  const Part mine = left[lane & (2 * NW - 1)];  // a part per lane
  unsigned todo = (unsigned)__ballot(lane < 2 * NW && mine.row >= 0);
  while (todo) {
    const int k0 = __ffs(todo) - 1, row = __builtin_amdgcn_readlane(mine.row, k0), n = __builtin_amdgcn_readlane(mine.n, k0);
    const unsigned set = todo & (unsigned)__ballot(mine.row == row);
    const int last = __builtin_amdgcn_readlane(mine.block1, 31 - __clz(set));
    todo &= ~set;
    const bool begins = __builtin_amdgcn_readlane(mine.block0, k0) == 0, whole = begins && last == n;
    const int64_t head0 = (int64_t)row * p.G + heads.first, part0 = part_at(p, group, begins) + heads.first;
    for (int i = tid; i < heads.n * D; i += NW * 64) {
      const int h = i / D;
      // all parts' numbers, whether they are the row's or not: what is not is left out by its factor
      float2 v[2 * NW];
      float x[2 * NW], M = -INFINITY;
#pragma unroll
      for (int k = 0; k < 2 * NW; ++k) {
        v[k] = ml[k][h];
        x[k] = acc[k * stride + i];
      }
#pragma unroll
      for (int k = 0; k < 2 * NW; ++k) {
        if (!(set >> k & 1)) v[k] = make_float2(-INFINITY, 0.f);
        M = fmaxf(M, v[k].x);
      }
      float a = 0.f, l = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * NW; ++k) {
        const float f = v[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((v[k].x - M) * cexp);
        a += v[k].x == -INFINITY ? 0.f : x[k] * f;
        l += v[k].y * f;
      }
      if (whole) {
        p.out[head0 * D + i] = l == 0.f ? 0.f : a / l;
        if (p.lse && i % D == 0) p.lse[head0 + h] = l == 0.f ? -INFINITY : fmaf(M, p.join_scale, logf(l));
      } else {
        p.part_acc[part0 * D + i] = a;
        if (i % D == 0) p.part_ml[part0 + h] = make_float2(M, l);
      }
    }
    // Where a row's parts lie is said by the workgroup that begins it: a record per row (of rows without tokens by clear_empty), or, where there are
    // more rows than workgroups, one per workgroup.
    if (tid == 0 && heads.first == 0 && begins && (!whole || p.by_row)) {
      JoinRecord r = {row, -1, 0};
      if (!whole) {
        r.first = group;
        r.last = shares.of(__builtin_amdgcn_readlane(mine.row_end, k0) - 1) / NW;
      }
      p.joins[p.by_row ? row : group] = r;
    }
  }
}

// Merges the parts of a row that were left in scratch: a workgroup per (record, head), or, where there are few parts, a wave per head.
template <int D>
__global__ __launch_bounds__(256) void join_kernel(CacheAttnParams p) {
  constexpr int C4 = D / 4, Q = 256 / C4, U = 8;  // lanes per part (16 bytes each), parts at a time, rounds in flight at the start
  __shared__ float factor[kAttnGroups];
  __shared__ float4 sums[Q][C4];
  __shared__ float s_max[4];
  __shared__ double s_den[4];
  const JoinRecord r = p.joins[blockIdx.x];
  // (the bounds are for lengths that changed under the call: a record that nobody wrote is whatever the workspace held)
  if (r.first < 0 || r.last < r.first || r.last >= kAttnGroups || (unsigned)r.row >= (unsigned)(p.P * p.Hkv)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = r.last - r.first + 1;
  const float c = p.join_scale * 1.44269502162933349609375f;
  auto finish = [&](int g, int j, float num, double den, float M) {  // dim j of head g
    const int64_t head = (int64_t)r.row * p.G + g;
    p.out[head * D + j] = den == 0.0 ? 0.f : num / (float)den;
    if (p.lse && j == 0) p.lse[head] = den == 0.0 ? -INFINITY : fmaf(M, p.join_scale, logf((float)den));
  };
  if (n <= U) {
    const int g = blockIdx.y * 4 + wave;
    if (g < p.G) {
      auto part = [&](int s) { return part_at(p, r.first + s, s == 0) + g; };
      const float2 v = lane < n ? p.part_ml[part(lane)] : make_float2(-INFINITY, 0.f);
      float2 a[U];
#pragma unroll
      for (int u = 0; u < U; ++u) a[u] = lane < D / 2 ? reinterpret_cast<const float2*>(p.part_acc + part(min(u, n - 1)) * D)[lane] : make_float2(0.f, 0.f);
      const float M = wave_combine<true, 1>(v.x);
      const float f = v.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((v.x - M) * c);
      const double den = group_sum_f64<64>((double)v.y * f);
      float2 num = make_float2(0.f, 0.f);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fu = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), u));  // 0 behind the last part
        if (fu == 0.f) continue;
        num.x = fmaf(a[u].x, fu, num.x);
        num.y = fmaf(a[u].y, fu, num.y);
      }
      if (lane < D / 2) {
        finish(g, 2 * lane, num.x, den, M);
        finish(g, 2 * lane + 1, num.y, den, M);
      }
    }
    return;
  }
  const int q = tid / C4, j = tid % C4, g = blockIdx.y;
  auto part = [&](int s) { return part_at(p, r.first + s, s == 0) + g; };
  auto acc = [&](int s) { return reinterpret_cast<const float4*>(p.part_acc)[part(s) * C4 + j]; };
  float4 early[U];
#pragma unroll
  for (int u = 0; u < U; ++u) early[u] = acc(min(q + u * Q, n - 1));
  float M = -INFINITY;
  for (int s = tid; s < n; s += 256) M = fmaxf(M, p.part_ml[part(s)].x);
  M = wave_combine<true, 1>(M);
  if (lane == 0) s_max[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  // the parts' factors; one without weight (all of its logits -infinity) is left out
  double den = 0.0;
  for (int s = tid; s < n; s += 256) {
    const float2 v = p.part_ml[part(s)];
    const float f = v.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((v.x - M) * c);
    factor[s] = f;
    den += (double)v.y * f;
  }
  den = group_sum_f64<64>(den);
  if (lane == 0) s_den[wave] = den;
  __syncthreads();
  den = (s_den[0] + s_den[1]) + (s_den[2] + s_den[3]);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& v, float f) {
    if (f == 0.f) return;
    a.x = fmaf(v.x, f, a.x), a.y = fmaf(v.y, f, a.y), a.z = fmaf(v.z, f, a.z), a.w = fmaf(v.w, f, a.w);
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (q + u * Q < n) add(early[u], factor[q + u * Q]);
  for (int s0 = q + U * Q; s0 < n; s0 += 4 * Q) {
    float4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = acc(min(s0 + u * Q, n - 1));
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u * Q < n) add(v[u], factor[s0 + u * Q]);
  }
  sums[q][j] = a;
  __syncthreads();
  if (tid < D) {
    float num = 0.f;
#pragma unroll
    for (int i = 0; i < Q; ++i) num += reinterpret_cast<const float*>(&sums[i][0])[tid];
    finish(g, tid, num, den, M);
  }
}

// bf16 caches.  A block of a wave: K goes through the wave's staging buffer in LDS (16-byte chunks, XOR-swizzled) into
// v_mfma_f32_16x16x32_bf16 with the queries as the A operand, their rows repeated, so that a lane takes the tile of its slot and ends
// with 4 logits of one token; V goes through the same buffer and is read transposed (ds_read_b64_tr_b16).  A softmax weight, fp32, is cut into three bf16
// parts of 8 bits each, which add up to it exactly: rows of the second product's A operand that the group's heads leave free take them, so up to four heads
// cost one product as they would with weights rounded to bf16, eight two, sixteen three.  (Rounded to bf16 the weights would put the outputs 1e-3 off, fp32's
// own error is 1e-6, and the matrix cores have nothing else to do: a workgroup's four blocks are 64 KB, which the CU's share of HBM brings in 2.4 us.)
//
// 8 rows of 524301 tokens, 4 heads, 128 dims: 321 us, 6.7 TB/s (7.1 to 7.4 is what reads alone reach); 256 rows of 1 to 32K tokens, 7 heads: 80 us, 5.2 TB/s; 8 rows of 32001: 30
// us, 4.4 TB/s.
template <int D, int GPAD>
__global__ __launch_bounds__(NW * 64, D == 64 && GPAD > 4 ? 1 : 2) void cache_attn_bf16_kernel(CacheAttnParams p) {
  constexpr int BT = attn_block(DT_BF16, D);
  constexpr int CH = D / 8, TPL = 64 / CH, NLOAD = BT / TPL, KSTEPS = D / 32;
  constexpr int TILES = 16 / GPAD, NT = BT / 16;     // tiles of 16 tokens a q.K accumulator has slots for, tiles of a block
  constexpr int NACC = NT > TILES ? NT / TILES : 1;  // q.K accumulators of a block
  constexpr int NDT = D / 16;                        // output tiles of 16 dims
  constexpr int NSET = GPAD == 4 ? 1 : GPAD == 8 ? 2 : 3;  // A operands of the second product
  // per wave: accumulators of its first part; staging buffer, at the end the accumulators of its last part.  (Part k's are at lds + k * kSpan.)
  constexpr int kSpan = BT * CH;  // 16-byte units
  static_assert(GPAD * D * 4 <= kSpan * 16, "a part's accumulators fit a staging buffer");
  __shared__ uint4 lds[NW][2][kSpan];
  __shared__ __attribute__((aligned(16))) unsigned short pT[NW][BT][NSET * 16];  // parts of the weights, [token][part, head]
  __shared__ float2 s_ml[2 * NW][GPAD];
  __shared__ Part s_left[2 * NW];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tq = lane / CH, cl = lane % CH;  // load role: token of a load, 16-byte chunk
  const int n = lane & 15, j = lane >> 4;    // MFMA role: column, row block / k-group
  const int number = blockIdx.x * NW + wave;
  const Heads heads(p);
  const int g0 = heads.first, gb = heads.n;
  if (tid == 0 && g0 == 0 && !p.by_row) p.joins[blockIdx.x].first = -1;
  if (lane < 2) s_left[2 * wave + lane].row = -1;
  const int empty = length_of(p, min((int)blockIdx.x, p.P - 1));
  Ahead<BT> ahead;
  const Shares shares = ahead.start(p, number, lane);
  ahead.it = -1, ahead.block0 = ahead.block1 = 0;
  ahead.step(p, lane);

  uint4* buf = lds[wave][1];
  // rows that no head's parts are in: 2^-126, which adds nothing (0 would make NaN of an infinite value)
#pragma unroll
  for (int i = 0; i < NSET * 16 * BT / 512; ++i)
    reinterpret_cast<uint4*>(&pT[wave][0][0])[i * 64 + lane] = make_uint4(0x00800080u, 0x00800080u, 0x00800080u, 0x00800080u);
  const int hbase = (4 * j) % GPAD, tslot = (4 * j) / GPAD;  // this lane's heads and tile among a q.K accumulator's rows
  const float cexp = p.scale * 1.44269502162933349609375f, slack = 10.f / cexp;
  auto vswz = [](int t) { return CH == 16 ? (((t & 3) << 1) | (((t >> 3) & 1) << 3)) : ((t & 3) << 1); };

  uint4 kv[NLOAD], vv[NLOAD], qa[KSTEPS];
  auto load_q = [&](int prob, int c) {
    const char* qrow = p.q + (((int64_t)prob * p.Hq + c * p.G + g0 + n % GPAD) * D + 8 * j) * 2;
#pragma unroll
    for (int kc = 0; kc < KSTEPS; ++kc) {
      qa[kc] = make_uint4(0u, 0u, 0u, 0u);
      if (n % GPAD < gb) qa[kc] = ld16(qrow + 64 * kc);
    }
  };
  auto load_k = [&] {
#pragma unroll
    for (int g = 0; g < BT / 16; ++g) {
      const auto at = ahead.keys(g);
#pragma unroll
      for (int i = 0; i < 16 / TPL; ++i) kv[g * (16 / TPL) + i] = load_token<true>(at, p.cache.ks_token, i * TPL + tq, cl * 16);
    }
  };
  auto load_v = [&] {
#pragma unroll
    for (int g = 0; g < BT / 16; ++g) {
      const auto at = ahead.values(g);
#pragma unroll
      for (int i = 0; i < 16 / TPL; ++i) vv[g * (16 / TPL) + i] = load_token<true>(at, p.cache.vs_token, i * TPL + tq, cl * 16);
    }
  };
  float m_run[4], l_part[4];
  f32x4_t acc[NDT];
  auto reset = [&] {
#pragma unroll
    for (int r = 0; r < 4; ++r) m_run[r] = -INFINITY, l_part[r] = 0.f;
#pragma unroll
    for (int nd = 0; nd < NDT; ++nd) acc[nd] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  };
  if (ahead.valid) {
    load_q(ahead.prob, ahead.c);
    load_k();
    load_v();
    reset();
  }
  while (ahead.valid) {
    const bool last = ahead.block0 + ahead.it + 1 == ahead.block1;  // of the part's blocks
    Part part;
    if (last) part = {ahead.prob * p.Hkv + ahead.c, ahead.block0, ahead.block1, ahead.row.n, ahead.row_end};
    const int t0 = ahead.token0();
    const Mask mask(p, ahead.row.len);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last block's reads of the buffer are done
#pragma unroll
    for (int i = 0; i < NLOAD; ++i) {
      const int t = i * TPL + tq;
      buf[t * CH + (cl ^ (t & (CH - 1)))] = kv[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const bool cut = mask.cuts(t0, BT);  // wave-uniform: some of the block's tokens are not attended
    if (cut) {  // V of those is not to be looked at
#pragma unroll
      for (int i = 0; i < NLOAD; ++i)
        if (!mask.at(t0 + i * TPL + tq)) vv[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    ahead.step(p, lane);  // (V of the present block is on its way already)
    if (ahead.valid) load_k();

    float x[NACC][4];
#pragma unroll
    for (int ts = 0; ts < NT; ++ts) {
      const int t = ts * 16 + n;
      f32x4_t d = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < KSTEPS; ++kc) {
        const uint4 bb = buf[t * CH + ((4 * kc + j) ^ (t & (CH - 1)))];
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, qa[kc]), __builtin_bit_cast(bf16x8_t, bb), d, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) x[ts / TILES][r] = ts % TILES == 0 || tslot == ts % TILES ? d[r] : x[ts / TILES][r];
    }
    if (last && ahead.valid) load_q(ahead.prob, ahead.c);
#pragma unroll
    for (int a = 0; a < NACC; ++a) {
      const int tile = a * TILES + tslot;
      const bool in = tile < NT && (!cut || mask.at(t0 + tile * 16 + n));
#pragma unroll
      for (int r = 0; r < 4; ++r) x[a][r] = in && hbase + r < gb ? x[a][r] : -INFINITY;
    }
    // Online softmax, once per (token, head), in units of the products.  The reference that a head's weights are relative to is raised to its maximum only when
    // a weight would pass 2^10: what is summed is fp32 with its own exponent, so nothing is lost.  Lanes with the same heads agree on it.
    bool over = false;
#pragma unroll
    for (int a = 0; a < NACC; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) over = over || x[a][r] > m_run[r] + slack;
    if (__ballot(over)) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float bm = x[0][r];
#pragma unroll
        for (int a = 1; a < NACC; ++a) bm = fmaxf(bm, x[a][r]);
        bm = group16_max(bm);
        if (GPAD <= 4) bm = swap16_max(bm);
        if (GPAD <= 8) bm = swap32_max(bm);
        const float mn = fmaxf(m_run[r], bm), corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run[r] - mn) * cexp);
        l_part[r] *= corr;
        m_run[r] = mn;
#pragma unroll
        for (int nd = 0; nd < NDT; ++nd) acc[nd][r] *= corr;  // row 4j + r belongs to head hbase + r whatever part it is
      }
    }
#pragma unroll
    for (int a = 0; a < NACC; ++a) {
      // A weight in three parts of 8 bits.  None may be 0 where V could be infinite, or their product would be NaN: so the weight's last bit is set and the low
      // part is kept from vanishing (2^-24 of the weight, and 2^-126).  (V of tokens that are not attended is 0.)
      uint32_t hi[4], mid[4], lo[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float w = x[a][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[a][r] - m_run[r]) * cexp);
        l_part[r] += w;
        const uint32_t u = __float_as_uint(w) | 1u;
        hi[r] = u & 0xFFFF0000u;
        const float rest = __uint_as_float(u) - __uint_as_float(hi[r]);
        mid[r] = __float_as_uint(rest) & 0xFFFF0000u;
        lo[r] = __float_as_uint(fmaxf(rest - __uint_as_float(mid[r]), 0x1p-126f));
      }
      auto pair = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); };  // their upper halves
      const int tile = a * TILES + tslot;
      if (tile < NT) {
        unsigned short* to = &pT[wave][tile * 16 + n][hbase];
        *reinterpret_cast<uint2*>(to) = make_uint2(pair(hi[0], hi[1]), pair(hi[2], hi[3]));
        *reinterpret_cast<uint2*>(to + GPAD) = make_uint2(pair(mid[0], mid[1]), pair(mid[2], mid[3]));
        *reinterpret_cast<uint2*>(to + 2 * GPAD) = make_uint2(pair(lo[0], lo[1]), pair(lo[2], lo[3]));
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // weights visible; q.K's reads of the buffer done
#pragma unroll
    for (int i = 0; i < NLOAD; ++i) {
      const int t = i * TPL + tq;
      buf[t * CH + (cl ^ vswz(t))] = vv[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (ahead.valid) load_v();

    // Transposed reads of LDS: lane s of 16 gives the address of 4 rows (dims) of token s / 4 and receives its own row (dim) of 4 tokens.
    typedef short v4s_t __attribute__((ext_vector_type(4)));
    auto transposed = [](const unsigned short* at, const unsigned short* at4) {  // tokens 8 j .. + 3 and the next four
      const v4s_t x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s_t*)at);
      const v4s_t x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s_t*)at4);
      struct { v4s_t a, b; } pair = {x0, x1};
      return __builtin_bit_cast(bf16x8_t, pair);
    };
    bf16x8_t pa[BT / 32][NSET];
#pragma unroll
    for (int kt = 0; kt < BT / 32; ++kt)
#pragma unroll
      for (int i = 0; i < NSET; ++i) {
        const int tu = 32 * kt + 8 * j + (n >> 2), at = 16 * i + (n & 3) * 4;
        pa[kt][i] = transposed(&pT[wave][tu][at], &pT[wave][tu + 4][at]);
      }
#pragma unroll
    for (int nd = 0; nd < NDT; ++nd) {
      const unsigned short* b16 = reinterpret_cast<const unsigned short*>(buf);
#pragma unroll
      for (int kt = 0; kt < BT / 32; ++kt) {
        const int tu = 32 * kt + 8 * j + (n >> 2);
        const int cch = (2 * nd + ((n & 3) >> 1)) ^ vswz(tu);  // vswz(tu) = vswz(tu + 4)
        const bf16x8_t vb = transposed(b16 + (tu * CH + cch) * 8 + (n & 1) * 4, b16 + ((tu + 4) * CH + cch) * 8 + (n & 1) * 4);
#pragma unroll
        for (int i = 0; i < NSET; ++i) acc[nd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[kt][i], vb, acc[nd], 0, 0, 0);
      }
    }

    if (!last) continue;
    // the part's totals: weights over the lanes that share a head, accumulators over the rows that hold its parts
    const bool whole = part.whole(), first = !whole && ahead.valid;
    const int k = 2 * wave + !first;
    if (!whole && lane == 0) s_left[k] = part;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float ls = group_sum<16>(l_part[r]);
      if (GPAD <= 4) ls = swap16_sum(ls);
      if (GPAD <= 8) ls = swap32_sum(ls);
      if (n == 0 && j < GPAD / 4) s_ml[k][hbase + r] = make_float2(m_run[r], ls);
    }
    float* s_acc = reinterpret_cast<float*>(lds[wave][!first]);  // [GPAD][D]
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int nd = 0; nd < NDT; ++nd)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float a = acc[nd][r];
        if (GPAD == 4) a = swap16_sum(a);
        if (GPAD <= 8) a = swap32_sum(a);
        acc[nd][r] = a;
      }
    if (4 * j < GPAD) {
#pragma unroll
      for (int nd = 0; nd < NDT; ++nd)
#pragma unroll
        for (int r = 0; r < 4; ++r) s_acc[(4 * j + r) * D + nd * 16 + n] = acc[nd][r];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (whole) write_row<D>(p, heads, part.row, lane, s_acc, s_ml[k]);
    reset();
  }
  __syncthreads();
  finish_group<D, GPAD>(p, heads, shares, s_left, reinterpret_cast<const float*>(&lds[0][0][0]), kSpan * 4, s_ml);
  if (g0 == 0) clear_empty(p, empty);
}

// fp32 caches.  Both products and the sums in fp64 (an fp32 logit of magnitude 100 would be off by 2.5e-5, and so would its softmax weight);
// fp64 and fp32 multiply-adds take the same four cycles.  Eight lanes share a token, a logit's eight parts are summed while
// heads and lanes change places, and lane s of the eight ends with head s's logit, whose weight it computes once and leaves in LDS for the lanes that
// hold V's chunks.  GB heads, at most 8.
template <int D, int GB>
__global__ __launch_bounds__(256, GB <= 4 ? 2 : 1) void cache_attn_f32_kernel(CacheAttnParams p) {
  constexpr int BT = D == 128 ? 16 : 32;
  constexpr int CH = D / 4;
  constexpr bool LATE_V = GB >= 4;             // V's block after the logits, not with K's: else registers spill
  constexpr int NG = BT / 8, NC = CH / 8;      // K: groups of 8 tokens, a lane's chunks of a token
  constexpr int TPL = 64 / CH, NV = BT / TPL;  // V: tokens per load, loads
  constexpr int GP = (GB + 1) / 2 * 2;         // weights of a token in LDS: whole 16-byte pairs
  __shared__ __attribute__((aligned(16))) double s_q[NW][GB * D];
  __shared__ __attribute__((aligned(16))) double pw[NW][BT][GP];
  __shared__ __attribute__((aligned(16))) float s_acc[2 * NW][GB * D];
  __shared__ float2 s_ml[2 * NW][GB];
  __shared__ Part s_left[2 * NW];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t8 = lane >> 3, sl = lane & 7;   // K role: token of a group, share of a token; head, once the logits are summed
  const int tq = lane / CH, cl = lane % CH;  // V role: token of a load, chunk
  const int number = blockIdx.x * NW + wave;
  const Heads heads(p);
  const int g0 = heads.first;
  if (tid == 0 && g0 == 0 && !p.by_row) p.joins[blockIdx.x].first = -1;
  if (lane < 2) s_left[2 * wave + lane].row = -1;
  const int empty = length_of(p, min((int)blockIdx.x, p.P - 1));
  Ahead<BT> ahead;
  const Shares shares = ahead.start(p, number, lane);
  ahead.it = -1, ahead.block0 = ahead.block1 = 0;
  ahead.step(p, lane);

  double* qd = s_q[wave];
  uint4 kv[NG][NC], vv[NV];
  auto load_k = [&] {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const auto at = ahead.keys(g / 2);
#pragma unroll
      for (int ch = 0; ch < NC; ++ch) kv[g][ch] = load_token<false>(at, p.cache.ks_token, g % 2 * 8 + t8, sl * 16 + ch * 128);
    }
  };
  auto load_v = [&] {
#pragma unroll
    for (int i = 0; i < NV; ++i) vv[i] = load_token<false>(ahead.values(i * TPL / 16), p.cache.vs_token, i * TPL % 16 + tq, cl * 16);
  };
  constexpr int NQ = (GB * D + 63) / 64;
  float qv[NQ];  // the next part's queries
  auto load_q = [&](int prob, int c) {
    const float* q = (const float*)p.q + (((int64_t)prob * p.Hkv + c) * p.G + g0) * D;
#pragma unroll
    for (int i = 0; i < NQ; ++i) qv[i] = i * 64 + lane < heads.n * D ? q[i * 64 + lane] : 0.f;
  };
  auto keep_q = [&] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < NQ; ++i) qd[i * 64 + lane] = (double)qv[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  float m = -INFINITY;  // of head sl
  double l = 0.0, acc[GB][4];
  auto reset = [&] {
    m = -INFINITY;
    l = 0.0;
#pragma unroll
    for (int g = 0; g < GB; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g][e] = 0.0;
  };
  if (ahead.valid) {
    load_q(ahead.prob, ahead.c);
    load_k();
    if (!LATE_V) load_v();
    reset();
    keep_q();
  }
  while (ahead.valid) {
    const bool last = ahead.block0 + ahead.it + 1 == ahead.block1;  // of the part's blocks
    Part part;
    if (last) part = {ahead.prob * p.Hkv + ahead.c, ahead.block0, ahead.block1, ahead.row.n, ahead.row_end};
    const int t0 = ahead.token0();
    const Mask mask(p, ahead.row.len);
    const bool cut = mask.cuts(t0, BT);
    double x[NG];  // of head sl, token 8 g + t8
#pragma unroll
    for (int gg = 0; gg < NG; gg += 2) {
#pragma unroll
      for (int hh = 0; hh < GB; hh += 4) {
        asm volatile("" ::: "memory");  // the queries are read again, not held for the other groups
        double a[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int h = 0; h < 4; ++h) a[u][h] = 0.0;
#pragma unroll
        for (int ch = 0; ch < NC; ++ch) {
          double kd[2][4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            kd[u][0] = (double)__uint_as_float(kv[gg + u][ch].x);
            kd[u][1] = (double)__uint_as_float(kv[gg + u][ch].y);
            kd[u][2] = (double)__uint_as_float(kv[gg + u][ch].z);
            kd[u][3] = (double)__uint_as_float(kv[gg + u][ch].w);
          }
#pragma unroll
          for (int h = 0; h < 4 && hh + h < GB; ++h) {
            const double* q = qd + (hh + h) * D + (ch * 8 + sl) * 4;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) a[u][h] = fma(kd[u][e], q[e], a[u][h]);
          }
        }
        // over the eight lanes of a token; lane s keeps head s
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const double r = eight_lane_sums<GB>(a[u], sl);
          x[gg + u] = hh == 0 || sl >= 4 ? r : x[gg + u];
        }
      }
    }
    if (LATE_V) load_v();
    ahead.step(p, lane);
    if (ahead.valid) load_k();

    // softmax weights, once per (token, head)
    float bm = -INFINITY;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const bool in = sl < GB && (!cut || mask.at(t0 + 8 * g + t8));
      x[g] = in ? x[g] * (1.0 / sqrt((double)D)) : -INFINITY;
      bm = fmaxf(bm, (float)x[g]);
    }
    bm = fmaxf(bm, dpp_f32<0x128>(bm));  // row_ror:8
    bm = swap32_max(swap16_max(bm));
    const float mn = fmaxf(m, bm);
    const float corr = mn == -INFINITY ? 1.f : exp_fast(m - mn);
    l *= (double)corr;
    m = mn;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last block's weights are read
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float w = x[g] == -INFINITY ? 0.f : exp_fast((float)(x[g] - (double)mn));
      l += (double)w;
      if (sl < GB) pw[wave][8 * g + t8][sl] = (double)w;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

    if (cut) {  // what is not attended is not to be looked at
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (!mask.at(t0 + i * TPL + tq)) vv[i] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int g = 0; g < GB; ++g) {
      const double f = (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(corr), g));
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g][e] *= f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const double v[4] = {(double)__uint_as_float(vv[i].x), (double)__uint_as_float(vv[i].y), (double)__uint_as_float(vv[i].z),
                           (double)__uint_as_float(vv[i].w)};
#pragma unroll
      for (int g = 0; g < GB; ++g) {
        const double w = pw[wave][i * TPL + tq][g];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[g][e] = fma(w, v[e], acc[g][e]);
      }
    }
    if (!LATE_V && ahead.valid) load_v();

    if (!last) continue;
    // the part's totals: over the lanes that share a chunk of V, and those that share a head
    if (ahead.valid) load_q(ahead.prob, ahead.c);
    const bool whole = part.whole(), first = !whole && ahead.valid;
    const int k = 2 * wave + !first;
    if (!whole && lane == 0) s_left[k] = part;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int g = 0; g < GB; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double a = acc[g][e];
        if (CH == 16) a += swap16_f64(a);
        a = swap32_sum_f64(a);
        if (tq == 0) s_acc[k][g * D + cl * 4 + e] = (float)a;
      }
    l += dpp_f64<0x128>(l);
    l += swap16_f64(l);
    l = swap32_sum_f64(l);
    if (lane < GB) s_ml[k][lane] = make_float2(m, (float)l);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (whole) write_row<D>(p, heads, part.row, lane, s_acc[k], s_ml[k]);
    reset();
    if (ahead.valid) keep_q();
  }
  __syncthreads();
  finish_group<D, GB>(p, heads, shares, s_left, &s_acc[0][0], GB * D, s_ml);
  if (g0 == 0) clear_empty(p, empty);
}

template <int D, int GB = 1>
void launch_f32(const CacheAttnParams& p, dim3 grid, hipStream_t s) {
  if constexpr (GB < 8) {
    if (p.heads > GB) return launch_f32<D, GB + 1>(p, grid, s);
  }
  hipLaunchKernelGGL((cache_attn_f32_kernel<D, GB>), grid, dim3(NW * 64), 0, s, p);
}

template <int D>
void launch_bf16(const CacheAttnParams& p, dim3 grid, hipStream_t s) {
  if (p.heads <= 4) hipLaunchKernelGGL((cache_attn_bf16_kernel<D, 4>), grid, dim3(NW * 64), 0, s, p);
  else if (p.heads <= 8) hipLaunchKernelGGL((cache_attn_bf16_kernel<D, 8>), grid, dim3(NW * 64), 0, s, p);
  else hipLaunchKernelGGL((cache_attn_bf16_kernel<D, 16>), grid, dim3(NW * 64), 0, s, p);
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnParams& p0, bool join, hipStream_t s) {
  // Groups of more heads than a workgroup takes: evenly over several, in one launch.  (us, launches one after the other and one launch: fp32, 16 heads, 300 tokens 33.1
  // 17.1, 524301 tokens x 8 rows 1774 1520; bf16, 32 heads, 32001 tokens 64.2 52.5, 524301 649 641: K and V are read again all the same.)  So are fewer heads
  // where the rows, at their longest, leave waves without work: the fewer heads, the sooner a block is done, and K and V are read again from the caches.  (us, a workgroup and
  // several, two rows: fp32, 64 dims, 8 heads, 261 tokens 16.9 9.4, 600 14.4 10.6, 8000 13.9 12.4, 2 heads 10.0 9.3, 10.6 10.4, 10.2 11.0; bf16, 128 dims, 16 heads, 261 13.3 11.1,
  // 600 15.2 12.3, 4000 13.5 12.4, 7 heads 11.5 11.0, 13.0 12.1, 12.2 12.4.)
  CacheAttnParams p = p0;
  const int most = p.dtype == DT_BF16 ? 16 : 8, least = p.dtype == DT_BF16 ? 4 : 1;
  const int n = max((p.G + most - 1) / most, min((p.G + least - 1) / least, kAttnWaves / p.n_waves));
  p.heads = (p.G + n - 1) / n;
  const unsigned groups = (unsigned)((p.n_waves + NW - 1) / NW);
  const dim3 all(groups, (unsigned)((p.G + p.heads - 1) / p.heads));
  if (p.dtype == DT_BF16) p.D == 128 ? launch_bf16<128>(p, all, s) : launch_bf16<64>(p, all, s);
  else p.D == 128 ? launch_f32<128>(p, all, s) : launch_f32<64>(p, all, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (!join) return hipSuccess;
  const dim3 grid((unsigned)(p.by_row ? p.P * p.Hkv : groups), (unsigned)p.G);
  if (p.D == 128) hipLaunchKernelGGL(join_kernel<128>, grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL(join_kernel<64>, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace sagekv
