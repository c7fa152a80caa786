// Rotary positions, alone or on the way of new tokens into the full cache.
//
// A wave takes one token: its position, its place and the page's table entry are wave-uniform, and lane j forms pair j's angle
// (at most 64 pairs), pos * f in turns, reduced in fp64 to [-1/2, 1/2], its cosine and sine in fp32.  They go through LDS to the lanes that need
// them, once per token for all heads.  Then a head's row is shared by the lanes in steps of 2 NP elements: NP pairs, or 2 NP elements
// to copy; 16-byte loads and stores where rotary_dim allows it (NP = 8 bf16, 4 fp32), single elements (NP = 1) where it
// does not.  Bound by HBM (prompts: every element read and written once) or by latency (single tokens).
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

// NP consecutive elements of a row in registers, as they are in memory.
template <int DT, int NP>
struct Part {
  uint4 u;
  __device__ __forceinline__ void load(const char* p) { u = ld16(p); }
  template <bool STREAM>
  __device__ __forceinline__ void store(char* p) const {
    if (STREAM) st16_stream(p, u);
    else st16(p, u);
  }
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
};
template <int DT>
struct Part<DT, 1> {
  uint32_t u;
  __device__ __forceinline__ void load(const char* p) { u = DT == DT_BF16 ? *(const uint16_t*)p : *(const uint32_t*)p; }
  template <bool>
  __device__ __forceinline__ void store(char* p) const {
    if (DT == DT_BF16) *(uint16_t*)p = (uint16_t)u;
    else *(uint32_t*)p = u;
  }
  __device__ __forceinline__ void get(float* f) const { f[0] = __uint_as_float(DT == DT_BF16 ? u << 16 : u); }
  __device__ __forceinline__ void set(const float* f) { u = DT == DT_BF16 ? pack_bf16(f[0], 0.f) & 0xFFFFu : __float_as_uint(f[0]); }
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

template <int DT, int NP, int D, bool STREAM>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  constexpr int EB = DT == DT_BF16 ? 2 : 4;
  constexpr int LPT = D / (2 * NP), HS = 64 / LPT;  // lanes a head's row is shared by; heads a wave takes at a time
  constexpr int U = NP == 1 ? 8 : 4;                // rounds of heads in flight
  __shared__ float2 turn[4][64];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t64 = (int64_t)blockIdx.x * 4 + wave;
  if (t64 >= p.n_tokens) return;
  const int t = (int)t64;

  // The token's rows are asked for early: what is done with them waits for its position, which is up to five memory round trips away (the problem's number,
  // its offsets, its length, the page).
  const int slot = lane / LPT, cl = lane % LPT;
  const bool rotates = cl * NP < p.r / 2;
  const bool halves = rotates && !p.pairs_layout;
  // this lane's two parts of a row, NP elements each: x[j..] and x[j + r/2..], or 2 NP consecutive ones
  const int at0 = (halves ? cl * NP : 2 * cl * NP) * EB, at1 = halves ? at0 + p.r / 2 * EB : at0 + NP * EB;
  const char* qs = p.q.base ? p.q.base + (int64_t)t * p.q.token : nullptr;
  const char *ks = p.k.base + (int64_t)t * p.k.token, *vs = p.v.base + (int64_t)t * p.v.token;
  const int first = qs ? 0 : p.Hq, all = p.Hq + 2 * p.Hkv;
  const int per = (all - first + (int)gridDim.y * HS - 1) / ((int)gridDim.y * HS) * HS;  // heads of this part of the grid
  const int h0 = first + blockIdx.y * per;
  Part<DT, NP> a[U], b[U];
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
  const double freq = lane < p.r / 2 ? p.freq[lane] : 0.0;
  load(h0);

  // the token's problem and place
  int prob = 0, place = 0;
  bool stored = false;
  if (p.Hkv) {
    int count = 1, i = 0;
    prob = t;
    if (p.offsets) {
      prob = search.find(p.offsets, p.P, t, lane);
      if (prob >= p.P || t < p.offsets[0]) return;  // nobody's row
      const int begin = p.offsets[prob];
      count = p.offsets[prob + 1] - begin;
      i = t - begin;
    }
    place = p.lens[prob] - count + i;
    stored = place >= 0 && place < p.capacity;
  }
  int64_t block = prob;
  if (stored && p.cache.table) {
    block = p.cache.table[(int64_t)prob * p.cache.pitch + (place >> p.cache.shift)];
    stored = block >= 0 && block < p.cache.n_blocks;
  }
  const int64_t in_block = place & (int)((1u << p.cache.shift) - 1u);

  // cosines and sines of the token's pairs
  if (lane < p.r / 2) {
    const int pos = p.positions ? p.positions[t] : place;
    const double turns = (double)pos * (freq * 0.15915494309189533577);  // 1 / (2 pi)
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[wave][lane] = make_float2(p.amplitude * c, p.amplitude * p.sign * s);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float cs[NP], sn[NP];
  if (rotates) {
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const float2 v = turn[wave][cl * NP + e];
      cs[e] = v.x;
      sn[e] = v.y;
    }
  }

  char* qd = p.q_out.base + (int64_t)t * p.q_out.token;
  char* kd = p.cache.K + block * p.cache.ks_block + in_block * p.cache.ks_token;
  char* vd = p.cache.V + block * p.cache.vs_block + in_block * p.cache.vs_token;
  const int h1 = min(stored ? all : p.Hq, h0 + per);
  for (int hb = h0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * HS + slot;
      if (h >= h1) continue;
      if (rotates && h < p.Hq + p.Hkv) {
        float x[NP], y[NP];
        a[u].get(x);
        b[u].get(y);
        if (NP > 1 && p.pairs_layout) {  // 2 NP consecutive elements: x, y hold the pairs' members in turn
          float z[2 * NP];
#pragma unroll
          for (int e = 0; e < NP; ++e) z[e] = x[e], z[NP + e] = y[e];
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            const float xe = z[2 * e] * cs[e] - z[2 * e + 1] * sn[e], ye = z[2 * e + 1] * cs[e] + z[2 * e] * sn[e];
            z[2 * e] = xe;
            z[2 * e + 1] = ye;
          }
          a[u].set(z);
          b[u].set(z + NP);
        } else {
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            const float xe = x[e] * cs[e] - y[e] * sn[e], ye = y[e] * cs[e] + x[e] * sn[e];
            x[e] = xe;
            y[e] = ye;
          }
          a[u].set(x);
          b[u].set(y);
        }
      }
      char* dst = h < p.Hq ? qd + h * p.q_out.head
                  : h < p.Hq + p.Hkv ? kd + (h - p.Hq) * p.cache.ks_head
                                     : vd + (h - p.Hq - p.Hkv) * p.cache.vs_head;
      a[u].template store<STREAM>(dst + at0);
      b[u].template store<STREAM>(dst + at1);
    }
    hb += U * HS;
    if (hb >= h1) break;
    load(hb);
  }
}

template <int DT, int NP, bool STREAM>
void launch_rotary_d(const RotaryParams& p, dim3 grid, hipStream_t s) {
  if (p.D == 128) hipLaunchKernelGGL((rotary_kernel<DT, NP, 128, STREAM>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((rotary_kernel<DT, NP, 64, STREAM>), grid, dim3(256), 0, s, p);
}

template <int DT, int NP>
hipError_t launch_rotary_n(const RotaryParams& p, hipStream_t s) {
  const int HS = 64 / (p.D / (2 * NP)), heads = (p.q.base ? p.Hq : 0) + 2 * p.Hkv, rounds = (heads + HS - 1) / HS;
  // few tokens: their heads over several waves (latency)
  const int64_t want = (1024 + p.n_tokens - 1) / p.n_tokens;
  const dim3 grid((unsigned)((p.n_tokens + 3) / 4), (unsigned)(want < rounds ? want : rounds));
  // Streaming stores from 48 MB written on: lines that stay in the caches to be written back cost the stream more than they save the next kernel.  us, plain and
  // streaming, the call alone and with a kernel behind it that reads all it wrote (bf16, 32 + 8 heads of 128 dims): 2048 tokens 12.7 12.0, 36.2 36.5; 4096 25 19, 61.5 63.1; 8192
  // 47.5 41, 110 114; 32768 158 147, 416 412; 24 prompts of 6532 tokens in all 40.5 28.1; 32767 tokens' queries (28 heads) 91 82.
  if constexpr (NP > 1) {
    if (p.n_tokens * heads * p.D * (DT == DT_BF16 ? 2 : 4) >= 48ll << 20) {
      launch_rotary_d<DT, NP, true>(p, grid, s);
      return hipGetLastError();
    }
  }
  launch_rotary_d<DT, NP, false>(p, grid, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, hipStream_t s) {
  // 16-byte parts: a half, or the rotated elements, have to end at a part's end
  if (p.dtype == DT_BF16) return p.r % 16 == 0 ? launch_rotary_n<DT_BF16, 8>(p, s) : launch_rotary_n<DT_BF16, 1>(p, s);
  return p.r % 8 == 0 ? launch_rotary_n<DT_F32, 4>(p, s) : launch_rotary_n<DT_F32, 1>(p, s);
}

}  // namespace sagekv
