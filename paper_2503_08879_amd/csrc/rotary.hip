// Rotary positions, alone or on the way of new tokens into the full cache.
//
// A wave takes one token (or four small ones, in equal shares of its lanes): its position, its place, the page's table entry; and lane j forms pair j's angle
// (at most 64 pairs), pos * f in turns, reduced in fp64 to [-1/2, 1/2], its cosine and sine in fp32.  They go through LDS to the lanes that need
// them, once per token for all heads.  Then a head's row is shared by its lanes in two 16-byte parts each, one in
// each half of the row, neighbouring lanes' parts side by side for every load and store.  Where a pair's other member is, is the MODE:
//   HALVES  pairs (j, j + d/2) of whole rows: both members with one lane (rows that are only copied come here too);
//   PAIRS   pairs (2j, 2j + 1), r any: a part is whole pairs;
//   APART   pairs (j, j + r/2), r < d: a lane's elements find their other members in the row's copy in LDS.
// (us: two consecutive parts per lane in PAIRS 105 instead of 84, for 32767 tokens of 28 heads of 128 dims, bf16; a pair's members with one lane where r = 64, so that
// loads and stores are in pieces of 64 bytes, 93 instead of 89; single elements instead of parts where r = 20, for a prompt of 131072 tokens, 32 + 8 heads, 1009 instead of 579.)
//
// Stores are streaming ones: what stays in the caches has to be written back when the kernel ends, which nothing overlaps.  us, plain and streaming, 32 heads of 128
// dims, bf16: 512 tokens 5.5 5.3, 2048 10.5 7.3, 4096 14.0 13.8, 8192 29.0 28.3; with a kernel behind it that reads all that was written 10.1 10.1, 16.8 16.9, 27.0 25.9, 52.1 50.4; 24
// prompts of 6532 tokens in all, with their keys and values, 38.1 25.9; a layer's write and attention of one token each of 64 sequences the same.
//
// Bound by HBM (prompts: every element read and written once; 131072 tokens of 32 + 8 heads of 128 dims, bf16, 568 us, 5.7 TB/s) or by latency (a token 2.8 us).
#include "device_utils.h"
#include "full_cache.h"

namespace sagekv {

namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// two fp32 values rounded to bf16, to nearest even, NaN kept
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}

enum { HALVES, PAIRS, APART };

// 16 bytes of a row in registers, as they are in memory: N elements.
template <int DT>
struct Part {
  static constexpr int N = DT == DT_BF16 ? 8 : 4;
  uint4 u;
  __device__ __forceinline__ void load(const char* p) { u = ld16(p); }
  __device__ __forceinline__ void store(char* p) const { st16_stream(p, u); }
  __device__ __forceinline__ void get(float* f) const {
    if (DT == DT_BF16) {
      unpack16(u, f);
    } else {
      f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
    }
  }
  __device__ __forceinline__ void set(const float* f) {
    if (DT == DT_BF16)
      u = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else
      u = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  // the first n elements (an even number) set, the others as they are
  __device__ __forceinline__ void set_first(const float* f, int n) {
    const uint4 old = u;
    constexpr int E = DT == DT_BF16 ? 2 : 1;  // elements of 4 bytes
    set(f);
    u.x = n > 0 ? u.x : old.x;
    u.y = n > E ? u.y : old.y;
    u.z = n > 2 * E ? u.z : old.z;
    u.w = n > 3 * E ? u.w : old.w;
  }
};

// How many of ends[1 .. P] are <= t: the problem that row t belongs to, P past the last.  64 probes at a time, one memory round trip each; the first of
// them is asked for before the rows are, so that it is not waited for behind them.
struct ProblemSearch {
  int step, probe;
  __device__ __forceinline__ void ask(const int32_t* ends, int lo, int n, int lane) {
    step = (n + 63) / 64;
    probe = ends[lo + min((lane + 1) * step, n)];
  }
  __device__ __forceinline__ int find(const int32_t* ends, int P, int t, int lane) {
    int lo = 0, n = P;
    for (;;) {
      const int m = __popcll(__ballot((lane + 1) * step <= n && probe <= t)) * step;
      lo += m;
      n = min(n - m, step - 1);
      if (n <= 0) return lo;
      ask(ends, lo, n, lane);
    }
  }
};

// T tokens per wave, next to each other, in equal shares of its lanes.
template <int DT, int MODE, int D, int T>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  constexpr int EB = DT == DT_BF16 ? 2 : 4, NP = Part<DT>::N;
  constexpr int LPT = D / (2 * NP), HS = 64 / T / LPT;  // lanes a head's row is shared by; heads of a token at a time
  constexpr int U = 4;                              // rounds of heads in flight
  __shared__ float2 turn[4][T][64];
  __shared__ uint4 copy[MODE == APART ? 4 : 1][MODE == APART ? 128 : 1];  // APART: a wave's rows

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t64 = ((int64_t)blockIdx.x * 4 + wave) * T;
  if (t64 >= p.n_tokens) return;
  const int t0 = (int)t64, k = lane / (64 / T), t = min(t0 + k, (int)p.n_tokens - 1);  // the wave's first token, which of them this lane's is
  bool real = t0 + k < p.n_tokens;

  // The token's rows are asked for early: what is done with them waits for its position, which is up to five memory round trips away (the problem's number,
  // its offsets, its length, the page).
  const int slot = lane % (64 / T) / LPT, cl = lane % LPT;
  const bool rotates = cl * NP < p.r;
  const int e0 = cl * NP, e1 = D / 2 + e0, half = p.r / 2;  // first elements of this lane's two parts of a row
  const int at0 = e0 * EB, at1 = e1 * EB;
  const char* qs = p.q.base ? p.q.base + (int64_t)t * p.q.token : nullptr;
  const char *ks = p.k.base + (int64_t)t * p.k.token, *vs = p.v.base + (int64_t)t * p.v.token;
  const int first = qs ? 0 : p.Hq, all = p.Hq + 2 * p.Hkv;
  const int per = (all - first + (int)gridDim.y * HS - 1) / ((int)gridDim.y * HS) * HS;  // heads of this part of the grid
  const int h0 = first + blockIdx.y * per;
  Part<DT> a[U], b[U];
  auto load = [&](int hb) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * HS + slot;
      if (h < min(all, h0 + per)) {
        const char* src = h < p.Hq ? qs + h * p.q.head
                          : h < p.Hq + p.Hkv ? ks + (h - p.Hq) * p.k.head
                                             : vs + (h - p.Hq - p.Hkv) * p.v.head;
        a[u].load(src + at0);
        b[u].load(src + at1);
      }
    }
  };
  ProblemSearch search = {1, 0};
  if (p.offsets) search.ask(p.offsets, 0, p.P, lane);
  // angle i * 64 + lane is pair `pair[i]` of token `of[i]`
  double freq[T];
  int of[T], pair[T];
#pragma unroll
  for (int i = 0; i < T; ++i) {
    of[i] = T == 1 || half == 0 ? 0 : (i * 64 + lane) / half;
    pair[i] = i * 64 + lane - of[i] * half;
    freq[i] = i * 64 + lane < T * half ? p.freq[pair[i]] : 0.0;
  }
  load(h0);

  // the token's problem and place
  int prob = 0, place = 0;
  bool stored = false;
  if (p.Hkv) {
    int count = 1, i = 0;
    prob = t;
    if (p.offsets) {
      const int prob0 = search.find(p.offsets, p.P, t0, lane);
      prob = prob0;
      if (T > 1) {  // the others' problems are that one or, rarely, later ones
        const int at = prob0 + 1 + lane, end = p.offsets[min(at, p.P)];
#pragma unroll
        for (int j = 1; j < T; ++j) {
          const int ended = __popcll(__ballot(at <= p.P && end <= t0 + j));
          int other = prob0 + ended;
          if (ended == 64) {  // many problems without tokens between them
            search.ask(p.offsets, 0, p.P, lane);
            other = search.find(p.offsets, p.P, t0 + j, lane);
          }
          prob = k == j ? other : prob;
        }
      }
      real = real && prob < p.P && t >= p.offsets[0];  // else it is nobody's row
      if (T == 1 && !real) return;
      prob = min(prob, p.P - 1);
      const int begin = p.offsets[prob];
      count = p.offsets[prob + 1] - begin;
      i = t - begin;
    }
    place = p.lens[prob] - count + i;
    stored = real && place >= 0 && place < p.capacity;
  }
  int64_t block = prob;
  if (stored && p.cache.table) {
    block = p.cache.table[(int64_t)prob * p.cache.pitch + (place >> p.cache.shift)];
    stored = block >= 0 && block < p.cache.n_blocks;
  }
  const int64_t in_block = place & (int)((1u << p.cache.shift) - 1u);

  // cosines and sines of the tokens' pairs
  if (p.r > 0) {
    const int pos = p.positions ? p.positions[t] : place;
#pragma unroll
    for (int i = 0; i < T; ++i) {
      if (i * 64 >= T * half) break;
      const int pos_i = T == 1 ? pos : __shfl(pos, of[i] * (64 / T));
      if (i * 64 + lane >= T * half) continue;
      const double turns = (double)pos_i * (freq[i] * 0.15915494309189533577);  // 1 / (2 pi)
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      turn[wave][of[i]][pair[i]] = make_float2(p.amplitude * c, p.amplitude * p.sign * s);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  // HALVES: of the pairs that both parts share; PAIRS: of the first part's, then the second's; APART: of the elements, sines with their signs
  constexpr int NC = MODE == APART ? 2 * NP : NP;
  float cs[NC], sn[NC];
  if (rotates) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = MODE == HALVES ? 0 : (i < NC / 2 ? e0 : e1) + (MODE == APART ? i % (NC / 2) : 0);
      const int j = MODE == HALVES ? e0 + i : MODE == PAIRS ? e / 2 + i % (NC / 2) : e < half ? e : e - half;
      const float2 v = turn[wave][k][min(j, 63)];  // (behind the last pair: not used)
      cs[i] = v.x;
      sn[i] = MODE == APART && e < half ? -v.y : v.y;
    }
  }

  char* qd = p.q_out.base + (int64_t)t * p.q_out.token;
  char* kd = p.cache.K + block * p.cache.ks_block + in_block * p.cache.ks_token;
  char* vd = p.cache.V + block * p.cache.vs_block + in_block * p.cache.vs_token;
  const int h1 = real ? min(stored ? all : p.Hq, h0 + per) : 0, last = T == 1 ? h1 : min(all, h0 + per);
  for (int hb = h0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * HS + slot;
      if (h >= h1) continue;
      if (rotates && h < p.Hq + p.Hkv) {
        float x[2][NP], y[2][NP];
        a[u].get(x[0]);
        b[u].get(x[1]);
        if (MODE == HALVES) {
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            y[0][e] = x[0][e] * cs[e] - x[1][e] * sn[e];
            y[1][e] = x[1][e] * cs[e] + x[0][e] * sn[e];
          }
          a[u].set(y[0]);
          b[u].set(y[1]);
        } else if (MODE == PAIRS) {
#pragma unroll
          for (int e = 0; e < 2 * NP; e += 2) {
            const float m = x[e / NP][e % NP], n = x[e / NP][e % NP + 1], c = cs[e / 2], s = sn[e / 2];
            y[e / NP][e % NP] = m * c - n * s;
            y[e / NP][e % NP + 1] = n * c + m * s;
          }
          a[u].set_first(y[0], p.r - e0);
          b[u].set_first(y[1], p.r - e1);
        } else {
          char* row = (char*)copy[wave] + lane / LPT * (D * EB);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          *(uint4*)(row + at0) = a[u].u;
          *(uint4*)(row + at1) = b[u].u;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int i = 0; i < 2 * NP; ++i) {
            const int e = (i < NP ? e0 : e1) + i % NP, o = e < half ? e + half : e - half;  // o < D also where e >= r
            const float other = DT == DT_BF16 ? __uint_as_float((uint32_t)((const uint16_t*)row)[o] << 16) : ((const float*)row)[o];
            y[i / NP][i % NP] = x[i / NP][i % NP] * cs[i] + other * sn[i];
          }
          a[u].set_first(y[0], p.r - e0);
          b[u].set_first(y[1], p.r - e1);
        }
      }
      char* dst = h < p.Hq ? qd + h * p.q_out.head
                  : h < p.Hq + p.Hkv ? kd + (h - p.Hq) * p.cache.ks_head
                                     : vd + (h - p.Hq - p.Hkv) * p.cache.vs_head;
      a[u].store(dst + at0);
      b[u].store(dst + at1);
    }
    hb += U * HS;
    if (hb >= last) break;
    load(hb);
  }
}

template <int DT, int MODE>
hipError_t launch_rotary_m(const RotaryParams& p, hipStream_t s) {
  const int HS = 64 / (p.D / (2 * Part<DT>::N)), heads = (p.q.base ? p.Hq : 0) + 2 * p.Hkv, rounds = (heads + HS - 1) / HS;
  // few tokens: their heads over several waves (latency)
  const int64_t want = (1024 + p.n_tokens - 1) / p.n_tokens;
  const dim3 grid((unsigned)((p.n_tokens + 3) / 4), (unsigned)(want < rounds ? want : rounds));
  // Tokens that fill at most half of a wave's lanes, and enough of them for all SIMDs: four per wave, so that the way to their places, five memory round trips, is gone
  // once for all.  (us, one and four tokens per wave, bf16: 160000 tokens of 4 + 2 heads, 64 dims 100 72, with 20 of them rotated 166 92; 16000 tokens' queries, 4 heads of 64 dims 8.5
  // 5.6; 32767, 4 heads of 128 dims 16.0 13.8; more than half: 8 heads of 128 dims 21.6 22.2, 160000 tokens of 16 + 1 heads of 128 dims 243 300.)
  if (heads <= HS / 2 && p.n_tokens >= 4096) {
    const dim3 fewer((unsigned)((p.n_tokens + 15) / 16));
    if (p.D == 128) hipLaunchKernelGGL((rotary_kernel<DT, MODE, 128, 4>), fewer, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((rotary_kernel<DT, MODE, 64, 4>), fewer, dim3(256), 0, s, p);
    return hipGetLastError();
  }
  // Tokens of 8 KB and more keep a wave's registers full of loads, and four workgroups per CU read and write faster than six or seven: LDS that nobody uses keeps others away.  (us,
  // bf16, 128 dims, seven, four and three workgroups: 131072 tokens of 32 + 8 heads 617 567 615, 16384 79.1 74.2 83.1, fp32 1259 1168 1235; smaller tokens, 32767 of 28 heads 85.6 86.5
  // 97.4, with 64 dims 45.2 48.7 56.1; fewer, whose last workgroups then run alone, 6532 of 32 + 8 heads 26 31.)
  const unsigned unused = p.n_tokens >= 16384 && p.D * heads * (16 / Part<DT>::N) >= 8192 ? 36000 - (MODE == APART ? 8192 : 0) : 0;
  if (p.D == 128) hipLaunchKernelGGL((rotary_kernel<DT, MODE, 128, 1>), grid, dim3(256), unused, s, p);
  else hipLaunchKernelGGL((rotary_kernel<DT, MODE, 64, 1>), grid, dim3(256), unused, s, p);
  return hipGetLastError();
}

template <int DT>
hipError_t launch_rotary_t(const RotaryParams& p, hipStream_t s) {
  if (p.r && p.pairs_layout) return launch_rotary_m<DT, PAIRS>(p, s);
  return p.r == 0 || p.r == p.D ? launch_rotary_m<DT, HALVES>(p, s) : launch_rotary_m<DT, APART>(p, s);
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, hipStream_t s) {
  return p.dtype == DT_BF16 ? launch_rotary_t<DT_BF16>(p, s) : launch_rotary_t<DT_F32>(p, s);
}

}  // namespace sagekv
