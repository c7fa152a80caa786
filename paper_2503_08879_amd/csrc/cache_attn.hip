// Attention of one new token per sequence over the full cache, every sequence of its own length.
//
// A row (sequence, KV head) is cut into blocks of 32 tokens.  All rows, one after the other, are divided over the launch's workgroups, whatever their
// lengths: a row weighs its blocks and kRowWeight more for its beginning and end, and every workgroup gets the same weight.  It finds its share from the
// lengths alone, which it reads on the device (64 of them at a time, summed over the wave).  A row that one workgroup has for itself is written straight
// to `out`; parts of a row shared by several go to scratch, at most two a workgroup: one that continues a row and one that begins
// one.  join_kernel merges them, (max, sum, accumulator) by (max, sum, accumulator).
//
// Bound by HBM: K and V are read once, for all heads of the group at a time.
#include "device_utils.h"
#include "full_cache.h"

namespace sagekv {

namespace {

// ---- rows, weights and shares ------------------------------------------------------------------
// Lengths do not change while a launch runs: through the constant address space they come by scalar loads, which nothing else waits for.  (A vector
// load of a length in the middle of a share waits for all of K and V that is in flight.)
__device__ __forceinline__ int length_of(const CacheAttnParams& p, int prob) {
  return ((const __attribute__((address_space(4))) int*)p.lens)[prob];
}

// The blocks of a row of len tokens that hold attended tokens.  With a window those of the first S and of the last W tokens.
struct RowBlocks {
  int len, n;      // tokens; blocks
  int head, skip;  // blocks from `head` on lie `skip` blocks further
  __device__ __forceinline__ int token(int block) const { return (block < head ? block : block + skip) * kBlock; }
};
__device__ __forceinline__ RowBlocks row_blocks(const CacheAttnParams& p, int len) {
  RowBlocks r;
  r.len = len < 0 ? 0 : len < p.max_len ? len : p.max_len;
  r.n = (r.len + kBlock - 1) / kBlock;
  r.head = r.n;
  r.skip = 0;
  if (p.W > 0) {
    const int head = (p.S + kBlock - 1) / kBlock, tail = (r.len - p.W) / kBlock;  // first block of the window
    if (r.len > p.W && tail > head) {
      r.head = head;
      r.skip = tail - head;
      r.n -= r.skip;
    }
  }
  return r;
}
__device__ __forceinline__ int weight_of(const CacheAttnParams& p, int blocks) {
  return blocks == 0 ? 0 : p.whole_rows ? 1 : blocks + kRowWeight;
}

// The shares: `more` of them of size + 1, the others of size.
struct Shares {
  int groups, size, more;
  __device__ __forceinline__ Shares(int total, int groups_) : groups(groups_), size(total / groups_), more(total - total / groups_ * groups_) {}
  __device__ __forceinline__ int begin(int group) const { return group * size + min(group, more); }
  __device__ __forceinline__ int group_of(int at) const {
    const int large = more * (size + 1);
    return at < large ? at / (size + 1) : more + (at - large) / size;
  }
};

// One row's part in a workgroup.
struct Segment {
  int prob, c, block0, block1;
  RowBlocks row;
  int row_end;  // in weights, from the first row's beginning
  __device__ __forceinline__ bool whole() const { return block0 == 0 && block1 == row.n; }
};

// A workgroup's rows in turn.
struct Walk {
  int at, end;  // its share, in weights
  int prob, c, done;  // the row that `at` is in, and what of its weight lies before
  RowBlocks row;
  // the next row's part that holds blocks; false: none is left
  __device__ __forceinline__ bool next(const CacheAttnParams& p, Segment* g) {
    while (at < end) {
      const int weight = weight_of(p, row.n);
      if (done == weight) {
        done = 0;
        if (++c == p.Hkv) {
          c = 0;
          do row = row_blocks(p, length_of(p, ++prob));
          while (row.n == 0 && prob + 1 < p.P);
        }
        continue;
      }
      const int take = min(weight - done, end - at);
      const int skip = p.whole_rows ? 0 : kRowWeight;
      g->prob = prob, g->c = c, g->row = row;
      g->row_end = at - done + weight;
      g->block0 = max(done - skip, 0);
      g->block1 = p.whole_rows ? row.n : max(done + take - skip, 0);
      at += take;
      done += take;
      if (g->block1 > g->block0) return true;
    }
    return false;
  }
};

__device__ __forceinline__ int weights_of(const CacheAttnParams& p, int first, int n) {
  int sum = 0;
  for (int i0 = 0; i0 < n; i0 += 4) {
    int len[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) len[i] = p.lens[first + min(i0 + i, n - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += i0 + i < n ? weight_of(p, row_blocks(p, len[i]).n) : 0;
  }
  return sum;
}
__device__ __forceinline__ void find_share(const CacheAttnParams& p, int group, int lane, Walk* w, Shares* shares) {
  int lo = 0, n = p.P, before = 0;
  bool counted = false;
  for (;;) {  // a problem out of 64, of 64 * 64, ...
    const int per = (n + 63) / 64, first = lane * per, mine = max(0, min(per, n - first));
    const int incl = wave_scan_incl(weights_of(p, lo + first, mine)) * p.Hkv;
    if (!counted) {
      counted = true;
      const int total = __builtin_amdgcn_readlane(incl, 63);
      const int busy = p.whole_rows ? total : (total + kGroupBlocks - 1) / kGroupBlocks;
      *shares = Shares(total, max(1, min(busy, p.n_groups)));
      w->at = w->end = 0;
      if (group >= shares->groups || total == 0) return;
      w->at = shares->begin(group);
      w->end = shares->begin(group + 1);
    }
    // the first lane whose problems reach beyond the share's begin
    const int hit = __ffsll((unsigned long long)__ballot(before + incl > w->at)) - 1;
    before += hit > 0 ? __builtin_amdgcn_readlane(incl, hit - 1) : 0;
    lo += hit * per;
    n = min(per, n - hit * per);
    if (per == 1) break;
  }
  w->prob = lo;
  w->row = row_blocks(p, length_of(p, lo));
  const int weight = weight_of(p, w->row.n), in_problem = w->at - before;
  w->c = in_problem / weight;
  w->done = in_problem - w->c * weight;
}

// Where a row's parts lie, left by the workgroup that begins the row: a record per row (of rows without tokens by clear_empty), or, where there
// are more rows than workgroups, one per workgroup, which begins one row at most that it does not end.
__device__ __forceinline__ void leave_record(const CacheAttnParams& p, const Shares& shares, const Segment& g, int group) {
  const int row = g.prob * p.Hkv + g.c;
  if (g.block0 != 0 || (g.whole() && !p.by_row)) return;
  JoinRecord r = {row, -1, 0};
  if (!g.whole()) {
    r.first = group;
    r.last = shares.group_of(g.row_end - 1);
  }
  p.joins[p.by_row ? row : group] = r;
}

// Problems without tokens: out = 0, lse = -infinity.
__device__ __forceinline__ void clear_empty(const CacheAttnParams& p) {
  for (int prob = blockIdx.x; prob < p.P; prob += gridDim.x) {
    if (length_of(p, prob) > 0) continue;
    for (int i = threadIdx.x; i < p.Hq * p.D; i += blockDim.x) p.out[(int64_t)prob * p.Hq * p.D + i] = 0.f;
    if (p.lse)
      for (int i = threadIdx.x; i < p.Hq; i += blockDim.x) p.lse[(int64_t)prob * p.Hq + i] = -INFINITY;
    if (p.by_row)
      for (int c = threadIdx.x; c < p.Hkv; c += blockDim.x) p.joins[prob * p.Hkv + c].first = -1;
  }
}

// Tokens of a row that are attended; a block of n tokens from t0 on: are there any that are not?
struct Mask {
  int len, S, tail;  // tokens t < S or t >= tail, and t < len
  __device__ __forceinline__ Mask(const CacheAttnParams& p, int len_) : len(len_), S(p.S), tail(p.W > 0 ? len_ - p.W : 0) {}
  __device__ __forceinline__ bool at(int t) const { return t < len && (t < S || t >= tail); }
  __device__ __forceinline__ bool cuts(int t0, int n) const { return t0 + n > len || (tail > t0 && t0 + n > S); }
};

// Loads of a wave, in the order of its blocks, segment after segment: its it-th block of a segment is the segment's block
// wave + NW * it.  They run a block ahead of the arithmetic, into the next row's first block too: the merge of a row's waves would otherwise leave the memory idle.
template <int D, int NW>
struct BlockLoads {
  static constexpr int CH = D / 8, TPL = 64 / CH, NLOAD = kBlock / TPL;
  Walk walk;
  RowBlocks row;
  int wave, lane, prob, c, first, n, it;
  int pages;  // of the next 64 groups of 16 tokens, one per lane (a dense cache's "page" is the problem)
  bool valid;
  __device__ __forceinline__ BlockLoads(const CacheAttnParams& p, const Walk& w, int wave_, int lane_)
      : walk(w), wave(wave_), lane(lane_), n(0), it(-1), valid(true) {
    step(p);
  }
  // to the next block; valid: there is one
  __device__ __forceinline__ void step(const CacheAttnParams& p) {
    ++it;
    while (it >= n) {
      Segment g;
      valid = walk.next(p, &g);
      if (!valid) return;
      row = g.row, prob = g.prob, c = g.c;
      first = g.block0 + wave;
      n = g.block1 > first ? (g.block1 - first + NW - 1) / NW : 0;
      it = 0;
    }
    if ((it & 31) != 0) return;
    pages = prob;
    if (!p.cache.table) return;
    const int t = min(row.token(first + min(it + (lane >> 1), n - 1) * NW) + (lane & 1) * 16, row.len - 1);
    const int page = p.cache.table[(int64_t)prob * p.cache.pitch + (t >> p.cache.shift)];
    pages = page < 0 ? 0 : page >= p.cache.n_blocks ? p.cache.n_blocks - 1 : page;
  }
  // Tokens behind the row are its last one again.
  __device__ __forceinline__ void load(const CacheAttnParams& p, const char* base, int64_t s_block, int64_t s_head, int64_t s_token, uint4 (&dst)[NLOAD]) const {
    const int t0 = row.token(first + it * NW), in_block = (int)((1u << p.cache.shift) - 1u);
    base += c * s_head;
#pragma unroll
    for (int i = 0; i < NLOAD; ++i) {
      const char* b = base + (int64_t)__builtin_amdgcn_readlane(pages, (it * 2 + i * TPL / 16) & 63) * s_block;
      const int t = min(t0 + i * TPL + lane / CH, row.len - 1) & in_block;
      dst[i] = ld16_stream(b + t * s_token + lane % CH * 16);
    }
  }
  __device__ __forceinline__ void load_k(const CacheAttnParams& p, uint4 (&dst)[NLOAD]) const {
    load(p, p.cache.K, p.cache.ks_block, p.cache.ks_head, p.cache.ks_token, dst);
  }
  __device__ __forceinline__ void load_v(const CacheAttnParams& p, uint4 (&dst)[NLOAD]) const {
    load(p, p.cache.V, p.cache.vs_block, p.cache.vs_head, p.cache.vs_token, dst);
  }
};

// Merges the parts of a row that were left in scratch: a workgroup per (record, head).
__global__ __launch_bounds__(128) void join_kernel(CacheAttnParams p) {
  const JoinRecord r = p.joins[blockIdx.x];
  if (r.first < 0) return;
  const int g = blockIdx.y, j = threadIdx.x, sl = threadIdx.x & 31;
  if (j >= p.D) return;  // wave-uniform
  const int n = r.last - r.first + 1;
  auto part = [&](int s) { return ((int64_t)(r.first + s) * 2 + (s == 0)) * p.G + g; };
  float M = -INFINITY, num = 0.f;
  double den = 0.0;
  const float c = p.join_scale * 1.44269502162933349609375f;
  for (int s0 = 0; s0 < n; s0 += 32) {
    float2 v = make_float2(-INFINITY, 0.f);
    if (s0 + sl < n) v = p.part_ml[part(s0 + sl)];
    float av[32];
#pragma unroll
    for (int u = 0; u < 32; ++u) av[u] = s0 + u < n ? p.part_acc[part(s0 + u) * p.D + j] : 0.f;
    const float Mn = fmaxf(M, swap16_max(row_combine<true, 1>(v.x)));  // both halves of the wave hold the same 32 parts
    if (Mn == -INFINITY) continue;
    const float f = v.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((v.x - Mn) * c);
    const float f0 = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((M - Mn) * c);
    den = den * f0 + group_sum_f64<32>((double)v.y * f);
    num *= f0;
#pragma unroll
    for (int u = 0; u < 32; ++u)
      num = fmaf(av[u], __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), u)), num);
    M = Mn;
  }
  const int64_t head = (int64_t)r.row * p.G + g;
  p.out[head * p.D + j] = den == 0.0 ? 0.f : num / (float)den;
  if (p.lse && j == 0) p.lse[head] = den == 0.0 ? -INFINITY : fmaf(M, p.join_scale, logf((float)den));
}

// bf16 caches.  A wave takes 32 tokens at a time: K goes through the wave's staging buffer in LDS (16-byte chunks, XOR-swizzled) into
// v_mfma_f32_16x16x32_bf16 with the queries as the A operand, their rows repeated, so that a lane takes the tile of its slot and ends
// with 4 logits of one token; V goes through the same buffer and is read transposed (ds_read_b64_tr_b16).  A softmax weight, fp32, is cut into three bf16
// parts of 8 bits each, which add up to it exactly: rows of the second product's A operand that the group's heads leave free take them, so up to four heads
// cost one product as they would with weights rounded to bf16, eight two, sixteen three.  (Rounded to bf16 the weights would put the outputs 1e-3 off, fp32's
// own error is 1e-6, and the matrix cores have nothing else to do: four blocks of 128 dims are 64 KB, 2.5 us of HBM time for a CU.)
template <int D, int GPAD>
__global__ __launch_bounds__(256, 2) void cache_attn_bf16_kernel(CacheAttnParams p) {
  constexpr int BT = 32, NW = 4;
  constexpr int CH = D / 8, TPL = 64 / CH, NLOAD = BT / TPL, KSTEPS = D / 32, ROWB = D * 2;
  constexpr int TILES = 16 / GPAD, NT = BT / 16;     // tiles of 16 tokens a q.K accumulator has slots for, tiles of a block
  constexpr int NACC = NT > TILES ? NT / TILES : 1;  // q.K accumulators of a block
  constexpr int NDT = D / 16;                        // output tiles of 16 dims
  constexpr int NSET = GPAD == 4 ? 1 : GPAD == 8 ? 2 : 3;  // A operands of the second product
  static_assert(GPAD * D * 4 <= BT * ROWB, "a wave's accumulators fit its staging buffer");
  __shared__ uint4 kbuf[NW][BT * CH];
  __shared__ __attribute__((aligned(16))) unsigned short pT[NW][NSET * 16][BT];  // parts of the weights, [part, head][token]
  __shared__ float2 s_ml[NW][GPAD];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tq = lane / CH, cl = lane % CH;  // load role: token of a load, 16-byte chunk
  const int n = lane & 15, j = lane >> 4;    // MFMA role: column, row block / k-group
  const int group = blockIdx.x, g0 = p.g0, gb = p.gb;
  if (g0 == 0) clear_empty(p);
  if (tid == 0 && !p.by_row) p.joins[group].first = -1;
  Walk walk;
  Shares shares(0, 1);
  find_share(p, group, lane, &walk, &shares);
  BlockLoads<D, NW> ahead(p, walk, wave, lane);
  Segment seg;
  if (!walk.next(p, &seg)) return;

  uint4* buf = kbuf[wave];
#pragma unroll
  for (int i = 0; i < NSET; ++i) reinterpret_cast<uint4*>(&pT[wave][16 * i][0])[lane] = make_uint4(0u, 0u, 0u, 0u);  // rows nobody writes stay 0
  const int hbase = (4 * j) % GPAD, tslot = (4 * j) / GPAD;  // this lane's heads and tile among a q.K accumulator's rows
  const float cexp = p.scale * 1.44269502162933349609375f;
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
  load_q(seg.prob, seg.c);
  if (ahead.valid) {
    ahead.load_k(p, kv);
    ahead.load_v(p, vv);
  }
  for (;;) {
    const Mask mask(p, seg.row.len);
    const int first = seg.block0 + wave, nblk = seg.block1 > first ? (seg.block1 - first + NW - 1) / NW : 0;

    float m_run[4], l_part[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) m_run[r] = -INFINITY, l_part[r] = 0.f;
    f32x4_t acc[NDT];
#pragma unroll
    for (int nd = 0; nd < NDT; ++nd) acc[nd] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    for (int it = 0; it < nblk; ++it) {
      const int t0 = seg.row.token(first + it * NW);
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
      ahead.step(p);  // (V of the present block is on its way already)
      if (ahead.valid) ahead.load_k(p, kv);

      float x[NACC][4];
#pragma unroll
      for (int ts = 0; ts < NT; ++ts) {
        const int t = ts * 16 + n;
        f32x4_t d = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KSTEPS; ++kc) {
          const uint4 bb = buf[t * CH + ((4 * kc + j) ^ (n & (CH - 1)))];
          d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, qa[kc]), __builtin_bit_cast(bf16x8_t, bb), d, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) x[ts / TILES][r] = ts % TILES == 0 || tslot == ts % TILES ? d[r] : x[ts / TILES][r];
      }
#pragma unroll
      for (int a = 0; a < NACC; ++a) {
        const int tile = a * TILES + tslot;
        const bool in = tile < NT && (!cut || mask.at(t0 + tile * 16 + n));
#pragma unroll
        for (int r = 0; r < 4; ++r) x[a][r] = in && hbase + r < gb ? x[a][r] : -INFINITY;
      }
      // online softmax, once per (token, head), in units of the products; lanes with the same heads agree on the maximum
      float corr[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float bm = x[0][r];
#pragma unroll
        for (int a = 1; a < NACC; ++a) bm = fmaxf(bm, x[a][r]);
        bm = group16_max(bm);
        if (GPAD <= 4) bm = swap16_max(bm);
        if (GPAD <= 8) bm = swap32_max(bm);
        const float mn = fmaxf(m_run[r], bm);
        corr[r] = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_run[r] - mn) * cexp);
        float lsum = 0.f;
#pragma unroll
        for (int a = 0; a < NACC; ++a) {
          const float w = x[a][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x[a][r] - mn) * cexp);
          lsum += w;
          const int tile = a * TILES + tslot;
          if (tile < NT) {
            // three parts of 8 bits; one that is 0 beside a weight that is not becomes bf16's smallest number, so that an infinite value's product
            // with it is no NaN
            const uint32_t hi = __float_as_uint(w) & 0xFFFF0000u;
            const float rest = w - __uint_as_float(hi);
            uint32_t mid = __float_as_uint(rest) & 0xFFFF0000u;
            uint32_t lo = __float_as_uint(rest - __uint_as_float(mid));
            if (hi != 0u) {
              mid = mid == 0u ? 0x10000u : mid;
              lo = (lo >> 16) == 0u ? 0x10000u : lo;
            }
            const int col = tile * 16 + n;
            pT[wave][hbase + r][col] = (unsigned short)(hi >> 16);
            pT[wave][GPAD + hbase + r][col] = (unsigned short)(mid >> 16);
            pT[wave][2 * GPAD + hbase + r][col] = (unsigned short)(lo >> 16);
            if (GPAD == 8) pT[wave][3 * GPAD + hbase + r][col] = hi != 0u;  // beside the lows: no 0 there either
          }
        }
        l_part[r] = l_part[r] * corr[r] + lsum;
        m_run[r] = mn;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // weights visible; q.K's reads of the buffer done
#pragma unroll
      for (int i = 0; i < NLOAD; ++i) {
        const int t = i * TPL + tq;
        buf[t * CH + (cl ^ vswz(t))] = vv[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (ahead.valid) ahead.load_v(p, vv);

      uint4 pa[NSET];
#pragma unroll
      for (int i = 0; i < NSET; ++i) pa[i] = *reinterpret_cast<const uint4*>(&pT[wave][16 * i + n][8 * j]);
#pragma unroll
      for (int nd = 0; nd < NDT; ++nd) {
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[nd][r] *= corr[r];  // row 4j + r belongs to head hbase + r whatever part it is
        // transposed read: lane s of 16 gives the address of 4 dims of token s / 4 and receives its own dim of 4 tokens
        typedef short v4s_t __attribute__((ext_vector_type(4)));
        const int tu = 8 * j + (n >> 2);
        const int cch = (2 * nd + ((n & 3) >> 1)) ^ vswz(tu);  // vswz(tu) = vswz(tu + 4)
        const unsigned short* b16 = reinterpret_cast<const unsigned short*>(buf);
        const v4s_t x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4s_t*)(b16 + (tu * CH + cch) * 8 + (n & 1) * 4));
        const v4s_t x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4s_t*)(b16 + ((tu + 4) * CH + cch) * 8 + (n & 1) * 4));
        struct { v4s_t a, b; } pair = {x0, x1};
        const uint4 vb = __builtin_bit_cast(uint4, pair);
#pragma unroll
        for (int i = 0; i < NSET; ++i)
          acc[nd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, pa[i]), __builtin_bit_cast(bf16x8_t, vb), acc[nd], 0, 0, 0);
      }
    }

    Segment next;
    const bool more = walk.next(p, &next);
    if (more) load_q(next.prob, next.c);
    // the wave's totals: weights over the lanes that share a head, accumulators over the rows that hold its parts
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float ls = group_sum<16>(l_part[r]);
      if (GPAD <= 4) ls = swap16_sum(ls);
      if (GPAD <= 8) ls = swap32_sum(ls);
      if (n == 0 && j < GPAD / 4) s_ml[wave][hbase + r] = make_float2(m_run[r], ls);
    }
    float* s_acc = reinterpret_cast<float*>(buf);  // [GPAD][D]
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int nd = 0; nd < NDT; ++nd)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float a = acc[nd][r];
        if (GPAD == 4) {
          a = j < 3 ? a : 0.f;  // rows 12 to 15 are nobody's: 0 times a value that may be infinite
          a = swap16_sum(a);
        }
        if (GPAD <= 8) a = swap32_sum(a);
        if (4 * j < GPAD) s_acc[(4 * j + r) * D + nd * 16 + n] = a;
      }
    __syncthreads();
    constexpr int kAccStride = BT * ROWB / 4;  // floats between the waves' buffers
    const float* all = reinterpret_cast<const float*>(&kbuf[0][0]);
    const int64_t part = ((int64_t)group * 2 + (seg.block0 == 0)) * p.G + g0, head0 = ((int64_t)seg.prob * p.Hkv + seg.c) * p.G + g0;
#pragma unroll
    for (int i0 = 0; i0 < GPAD * D; i0 += NW * 64) {
      const int g = (i0 + tid) / D, jj = tid % D;
      if (g >= gb) break;
      float2 ml[NW];
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        ml[w] = s_ml[w][g];
        M = fmaxf(M, ml[w].x);
      }
      float a = 0.f, ls = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = ml[w].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[w].x - M) * cexp);
        a += ml[w].x == -INFINITY ? 0.f : all[w * kAccStride + g * D + jj] * f;
        ls += ml[w].y * f;
      }
      if (seg.whole()) {
        p.out[(head0 + g) * D + jj] = ls == 0.f ? 0.f : a / ls;
        if (p.lse && jj == 0) p.lse[head0 + g] = ls == 0.f ? -INFINITY : fmaf(M, p.scale, logf(ls));
      } else {
        p.part_acc[(part + g) * D + jj] = a;
        if (jj == 0) p.part_ml[part + g] = make_float2(M, ls);
      }
    }
    if (tid == 0) leave_record(p, shares, seg, group);
    if (!more) return;
    __syncthreads();  // buffers and s_ml are free again
    seg = next;
  }
}

// fp32 caches.  Both products and the sums in fp64 (an fp32 logit of magnitude 100 would be off by 2.5e-5, and so would its softmax weight);
// fp64 and fp32 multiply-adds take the same four cycles.  Eight lanes share a token, a logit's eight parts are summed while
// heads and lanes change places, and lane s of the eight ends with head s's logit, whose weight it computes once and leaves in LDS for the lanes that
// hold V's chunks.  GB heads, at most 8.
template <int D, int GB>
__global__ __launch_bounds__(D == 128 ? 512 : 256) void cache_attn_f32_kernel(CacheAttnParams p) {
  constexpr int NW = D == 128 ? 8 : 4, BT = kBlock * kGroupBlocks / NW, kThreads = NW * 64;
  constexpr int CH = D / 4, GPB = BT / 16;
  constexpr bool LATE_V = GB >= 4;             // V's block after the logits, not with K's: else registers spill
  constexpr int NG = BT / 8, NC = CH / 8;      // K: groups of 8 tokens, a lane's chunks of a token
  constexpr int TPL = 64 / CH, NV = BT / TPL;  // V: tokens per load, loads
  constexpr int GP = (GB + 1) / 2 * 2;         // weights of a token in LDS: whole 16-byte pairs
  __shared__ __attribute__((aligned(16))) double qd[GB * D];
  __shared__ __attribute__((aligned(16))) double pw[NW][BT][GP];
  __shared__ float s_acc[NW][GB][D];
  __shared__ float s_m[NW][GB];
  __shared__ double s_l[NW][GB];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t8 = lane >> 3, sl = lane & 7;   // K role: token of a group, share of a token; head, once the logits are summed
  const int tq = lane / CH, cl = lane % CH;  // V role: token of a load, chunk
  const int group = blockIdx.x, g0 = p.g0;
  if (g0 == 0) clear_empty(p);
  if (tid == 0 && !p.by_row) p.joins[group].first = -1;
  Walk walk;
  Shares shares(0, 1);
  find_share(p, group, lane, &walk, &shares);

  for (Segment seg; walk.next(p, &seg);) {
    const RowBlocks row = seg.row;
    const int prob = seg.prob, c = seg.c;
    const Mask mask(p, row.len);
    const int64_t head0 = ((int64_t)prob * p.Hkv + c) * p.G + g0;
    // 128 dims: two waves share a block
    constexpr int SHARE = kBlock / BT;
    auto token0 = [&](int it) { return row.token(seg.block0 + wave / SHARE + it * kGroupBlocks) + wave % SHARE * BT; };
    int nblk = (seg.block1 - seg.block0 - wave / SHARE + kGroupBlocks - 1) / kGroupBlocks;
    if (nblk > 0 && token0(nblk - 1) >= row.len) --nblk;

    const char* Kb = p.cache.K + c * p.cache.ks_head;
    const char* Vb = p.cache.V + c * p.cache.vs_head;
    const int32_t* tab = p.cache.table ? p.cache.table + (int64_t)prob * p.cache.pitch : nullptr;
    const int in_block = (int)((1u << p.cache.shift) - 1u);
    int my_block = prob;  // paged: pages of the wave's next 64 groups of 16 tokens, one per lane
    auto fill = [&](int it0) {
      if (!tab) return;
      const int it = min(it0 + lane / GPB, nblk - 1);
      const int t = min(token0(it) + lane % GPB * 16, row.len - 1);
      const int b = tab[t >> p.cache.shift];
      my_block = b < 0 ? 0 : b >= p.cache.n_blocks ? p.cache.n_blocks - 1 : b;
    };
    // token `base + of_lane` of block it, behind the row its last one
    auto address = [&](const char* at, int64_t s_block, int64_t s_token, int it, int base, int of_lane) {
      const int t = min(token0(it) + base + of_lane, row.len - 1);
      return at + (int64_t)__builtin_amdgcn_readlane(my_block, (it * GPB + base / 16) & 63) * s_block + (t & in_block) * s_token;
    };
    uint4 kv[NG][NC], vv[NV];
    auto load_k = [&](int it) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const char* a = address(Kb, p.cache.ks_block, p.cache.ks_token, it, 8 * g, t8) + sl * 16;
#pragma unroll
        for (int ch = 0; ch < NC; ++ch) kv[g][ch] = ld16(a + ch * 128);
      }
    };
    auto load_v = [&](int it) {
#pragma unroll
      for (int i = 0; i < NV; ++i) vv[i] = ld16(address(Vb, p.cache.vs_block, p.cache.vs_token, it, i * TPL, tq) + cl * 16);
    };
    if (nblk > 0) {
      fill(0);
      load_k(0);
      if (!LATE_V) load_v(0);
    }
    for (int i = tid; i < GB * D; i += kThreads) qd[i] = (double)((const float*)p.q)[head0 * D + i];
    __syncthreads();

    float m = -INFINITY;  // of head sl
    double l = 0.0, acc[GB][4];
#pragma unroll
    for (int g = 0; g < GB; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g][e] = 0.0;

    for (int it = 0; it < nblk; ++it) {
      const int t0 = token0(it);
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
      if (LATE_V) load_v(it);
      const bool more = it + 1 < nblk;
      if (more) {
        if ((((it + 1) * GPB) & 63) == 0) fill(it + 1);
        load_k(it + 1);
      }

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
      if (!LATE_V && more) load_v(it + 1);
    }

    // the wave's totals: over the lanes that share a chunk of V, and those that share a head
#pragma unroll
    for (int g = 0; g < GB; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double a = acc[g][e];
        if (CH == 16) a += swap16_f64(a);
        a = swap32_sum_f64(a);
        if (tq == 0) s_acc[wave][g][cl * 4 + e] = (float)a;
      }
    l += dpp_f64<0x128>(l);
    l += swap16_f64(l);
    l = swap32_sum_f64(l);
    if (lane < GB) {
      s_m[wave][lane] = m;
      s_l[wave][lane] = l;
    }
    __syncthreads();
    const int64_t part = ((int64_t)group * 2 + (seg.block0 == 0)) * p.G + g0;
    for (int i = tid; i < GB * D; i += kThreads) {
      const int g = i / D, jj = i % D;
      float M = s_m[0][g];
#pragma unroll
      for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w][g]);
      double a = 0.0, ls = 0.0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const double f = s_m[w][g] == -INFINITY ? 0.0 : (double)exp_fast(s_m[w][g] - M);
        a += s_m[w][g] == -INFINITY ? 0.0 : (double)s_acc[w][g][jj] * f;
        ls += s_l[w][g] * f;
      }
      if (seg.whole()) {
        p.out[(head0 + g) * D + jj] = ls == 0.0 ? 0.f : (float)(a / ls);
        if (p.lse && jj == 0) p.lse[head0 + g] = ls == 0.0 ? -INFINITY : (float)((double)M + log(ls));
      } else {
        p.part_acc[(part + g) * D + jj] = (float)a;
        if (jj == 0) p.part_ml[part + g] = make_float2(M, (float)ls);
      }
    }
    if (tid == 0) leave_record(p, shares, seg, group);
    __syncthreads();  // LDS is free again
  }
}

template <int D, int GB = 1>
void launch_f32(const CacheAttnParams& p, hipStream_t s) {
  if constexpr (GB < 8) {
    if (p.gb > GB) return launch_f32<D, GB + 1>(p, s);
  }
  hipLaunchKernelGGL((cache_attn_f32_kernel<D, GB>), dim3((unsigned)p.n_groups), dim3(D == 128 ? 512 : 256), 0, s, p);
}

template <int D>
void launch_bf16(const CacheAttnParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.n_groups);
  if (p.gb <= 4) hipLaunchKernelGGL((cache_attn_bf16_kernel<D, 4>), grid, dim3(256), 0, s, p);
  else if (p.gb <= 8) hipLaunchKernelGGL((cache_attn_bf16_kernel<D, 8>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((cache_attn_bf16_kernel<D, 16>), grid, dim3(256), 0, s, p);
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnParams& p, bool join, hipStream_t s) {
  CacheAttnParams q = p;
  const int per = p.dtype == DT_BF16 ? 16 : 8;  // heads a launch handles
  for (q.g0 = 0; q.g0 < p.G; q.g0 += per) {
    q.gb = p.G - q.g0 < per ? p.G - q.g0 : per;
    if (p.dtype == DT_BF16) p.D == 128 ? launch_bf16<128>(q, s) : launch_bf16<64>(q, s);
    else p.D == 128 ? launch_f32<128>(q, s) : launch_f32<64>(q, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!join) return hipSuccess;
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)(p.by_row ? p.P * p.Hkv : p.n_groups), (unsigned)p.G), dim3(128), 0, s, p);
  return hipGetLastError();
}

}  // namespace sagekv
