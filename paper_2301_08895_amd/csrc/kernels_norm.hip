// Group normalisation, channels last, with an activation behind it (abs_group_norm_*).
//
// What bounds it is memory: the forward pass has to read and write every element once, the backward pass to read x and dy
// and write dx.  So a group's values stay in registers between the statistics and their use wherever they fit:
//  * lanes go along the channels in pieces of V elements (16 bytes where the group width allows), a group's pieces padded
//    to a power of two of lanes (SP), several groups side by side (TX = SP gpc lanes: 128 bytes of a position and more, so
//    that lines are used whole) and PL positions on top: D = TX PL lanes hold one sample's share of gpc groups, NP
//    pieces each.  A workgroup holds T / D samples.
//  * a group's sum is then shuffles over powers of two, and, where D is more than a wavefront, one exchange through LDS.
//  * the variance is the mean of the squared distances from the mean, two passes over registers: nothing cancels.
// Samples that do not fit (and few large ones, which would leave most CUs idle) are cut into parts along the positions:
// one launch leaves each part's statistics, the next one joins them and writes.  Wide groups of single positions have kernels of their
// own (norm_row_kernel), and groups of more than 1024 pieces at several positions, or more than 4096 at one, a plain one.
#include "operators.h"

#include <algorithm>

namespace abs_impl {
namespace {

constexpr int kMaxLanes = 1024;            // D: lanes of one sample
constexpr int64_t kPlenty = 65536;         // lanes that fill the chip: 256 on a CU

template <typename T>
struct NormArgs {
  const T* x; const T* dy; const T* dres; T* y;          // y: dx in the backward pass
  const float* gamma; const float* beta;
  float* mean; float* rstd;                              // forward: outputs (may be null); backward: inputs
  int64_t n, S;
  int C, G, per, act;
  float eps;
  int64_t ldx, ldy, lddy, lddres;
  int slots, SP, gpc, TX, PL, D;                         // pieces of a group; lanes (see above)
  uint32_t chunks;                                       // of gpc groups
  uint32_t parts;                                        // of a sample
  int PP;                                                // positions of a part
  uint32_t work;                                         // workgroup's shares: (samples / samples of a workgroup) x parts x chunks
  float* part;                                           // [n][G][parts][2]: mean and squared distances, or the two sums
  float *rows_g, *rows_b;                                // backward: [row_count] shares of dgamma, dbeta, row_step floats apart (one share: theirs)
  int64_t row_step;
  uint32_t row_count;
};

// h = gamma rstd (x - mean) + beta, of the distance d = x - mean and s = gamma rstd: the same three roundings everywhere, so that a
// value at relu's corner is on the same side in every pass.
__device__ __forceinline__ float norm_h(float d, float s, float beta) { return fmaf(d, s, beta); }

// v + v of the lane whose number differs in bit OFF; kFlat: the lanes that differ in lower bits hold equal values already, so a
// mirror image does.  Cross-lane adds where there are such, swaps of rows or halves (which need no address either) and LDS's swizzle for
// the others.
template <int OFF, bool kFlat>
__device__ __forceinline__ float add_xor(float v) {
#define ABS_DPP(ctrl_) v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl_, 0xF, 0xF, true))
  if constexpr (OFF == 1) return ABS_DPP(0xB1);                        // quad_perm [1, 0, 3, 2]
  else if constexpr (OFF == 2) return ABS_DPP(0x4E);                   // quad_perm [2, 3, 0, 1]
  else if constexpr (OFF == 4 && kFlat) return ABS_DPP(0x141);         // row_half_mirror
  else if constexpr (OFF == 8 && kFlat) return ABS_DPP(0x140);         // row_mirror
  else if constexpr (OFF < 16) return v + __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(v), (OFF << 10) | 0x1F));
  else {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const unsigned u = (unsigned)__float_as_int(v);
    const u32x2 r = OFF == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);                // (even and odd rows, or the halves)
  }
#undef ABS_DPP
}
// ... over all bits that are set in `bits` (uniform)
template <bool kFlat>
__device__ __forceinline__ float add_lanes(float v, int bits) {
  asm volatile("" : "+s"(bits));          // (tested here: kept outside the loops, the tests' results would fill the scalar registers)
  if (bits & 1) v = add_xor<1, kFlat>(v);
  if (bits & 2) v = add_xor<2, kFlat>(v);
  if (bits & 4) v = add_xor<4, kFlat>(v);
  if (bits & 8) v = add_xor<8, kFlat>(v);
  if (bits & 16) v = add_xor<16, kFlat>(v);
  if (bits & 32) v = add_xor<32, kFlat>(v);
  return v;
}

// Sum of v over the lanes of one sample's group; every lane gets it.  `red`: 16 x 64 floats of LDS, not in use.
__device__ __forceinline__ float group_sum(float v, int SP, int TX, int D, float* red) {
  v = add_lanes<true>(v, SP - 1);                                      // pieces of the group
  v = add_lanes<false>(v, (D - 1) & ~(TX - 1));                        // positions
  if (SP > 64 || (D > 64 && D > TX)) {                                // (else a group is inside a wavefront)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int cols = SP < 64 ? min(TX, 64) / SP : 1;                  // groups of a wavefront
    if (SP < 64 ? (lane & (SP - 1)) == 0 && lane < min(TX, 64) : lane == 0) red[wave * 64 + (SP < 64 ? lane / SP : 0)] = v;
    __syncthreads();
    const int per_row = TX > 64 ? TX >> 6 : 1;                        // wavefronts of a position
    const int spread = SP > 64 ? SP >> 6 : 1;                         // ... of a group in it
    const int w0 = wave & ~((D >> 6) - 1);
    const int first = TX > 64 ? (wave & (per_row - 1)) & ~(spread - 1) : 0;
    const int col = SP < 64 ? (lane / SP) & (cols - 1) : 0;
    v = 0.f;
    for (int r = first; r < (D >> 6); r += per_row)
      for (int j = 0; j < spread; ++j) v += red[(w0 + r + j) * 64 + col];
  }
  return v;
}

// Where a thread stands: its sample inside the workgroup, positions p, p + PL, ..., group and piece.
// A group that is no whole number of pieces (TAIL) ends in one that has nv < V elements of its own.
struct Place {
  int sb, p, g, slot, nv;
  // how many of the lane's positions p, p + PL, ... lie below `positions`; none for a lane behind the group's pieces (the comparison of a
  // constant with this number is all that a piece costs: PL is a power of two, and positions kept for it would each take a register)
  template <typename A>
  __device__ __forceinline__ int pieces(int positions, const A& a) const {
    return p < positions && slot < a.slots ? ((positions - p - 1) >> (31 - __builtin_clz(a.PL))) + 1 : 0;
  }
};
template <typename T, int V, bool TAIL>
__device__ __forceinline__ Place place_of(const NormArgs<T>& a) {
  Place q;
  const int t = threadIdx.x, tx = t & (a.TX - 1);
  q.sb = t / a.D;
  q.p = (t & (a.D - 1)) / a.TX;
  q.g = tx / a.SP;
  q.slot = tx & (a.SP - 1);
  q.nv = TAIL ? min(V, a.per - q.slot * V) : V;
  return q;
}

// The last piece of a TAIL group is read V - nv elements early, so that it is one access inside the group, and moved down once it is there,
// zeros behind it.  (Only where everything is read before anything is written: the elements read twice may be another wavefront's to
// overwrite.)
template <typename T, int V>
__device__ __forceinline__ void move_down(Piece<T, V>& v, int nv) {
  const int skip = V - nv;
  if constexpr (sizeof(T) == 2 && V == 4) {
    const uint64_t x = (((uint64_t)v.w[1] << 32) | v.w[0]) >> (16 * skip);
    v.w[0] = (uint32_t)x; v.w[1] = (uint32_t)(x >> 32);
  } else if constexpr (sizeof(T) == 2) {
    v.w[0] >>= 16 * skip;
  } else {
    if (skip & 1) {
#pragma unroll
      for (int e = 0; e < V; ++e) v.w[e] = e + 1 < V ? v.w[e + 1] : 0;
    }
    if (V > 2 && skip & 2) {
#pragma unroll
      for (int e = 0; e < V; ++e) v.w[e] = e + 2 < V ? v.w[e + 2] : 0;
    }
  }
}
// ... or element by element; and what is written is its own elements alone.
template <bool TAIL, typename T, int V>
__device__ __forceinline__ void load_own(Piece<T, V>& v, const void* p, int nv) {
  if (!TAIL || nv == V) { v.load(p); return; }
  T e[V];
#pragma unroll
  for (int i = 0; i < V - 1; ++i) e[i] = ((const T*)p)[min(i, nv - 1)];       // (no branch, so that all are asked for at once)
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] = i < nv ? e[min(i, V - 2)] : T(0);
  __builtin_memcpy(v.w, e, V * sizeof(T));
}
template <bool TAIL, typename T, int V>
__device__ __forceinline__ void store_own(const Piece<T, V>& v, void* p, int nv) {
  if (!TAIL || nv == V) { v.store(p); return; }
  T e[V];
  __builtin_memcpy(e, v.w, V * sizeof(T));
#pragma unroll
  for (int i = 0; i < V - 1; ++i)
    if (i < nv) ((T*)p)[i] = e[i];
}
// gamma and beta of a piece's channels, from c on; 0 behind the group's end
template <bool TAIL, typename T, int V>
__device__ __forceinline__ void parameters(const NormArgs<T>& a, int c, int nv, float* gam, float* bet) {
#pragma unroll
  for (int e = 0; e < V; ++e) { gam[e] = 1.f; bet[e] = 0.f; }
  if (a.gamma) {
    Piece<float, V> pg, pb;
    if (TAIL) {
#pragma unroll
      for (int e = 0; e < V; ++e) { pg.w[e] = __float_as_uint(a.gamma[c + min(e, nv - 1)]); pb.w[e] = __float_as_uint(a.beta[c + min(e, nv - 1)]); }
    } else {
      pg.load(a.gamma + c);
      pb.load(a.beta + c);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) { gam[e] = e < nv ? pg.at(e) : 0.f; bet[e] = e < nv ? pb.at(e) : 0.f; }
  }
}

// Workgroup b of (samples x rest): neighbouring chunks of the same positions on one XCD (workgroups are dealt out over eight), one after
// the other: they share lines where a chunk is narrower than one.
__device__ __forceinline__ void place_work(uint32_t b, uint32_t per_sample, uint32_t samples, uint32_t& sample, uint32_t& rest) {
  const uint32_t whole = samples / 8 * 8;
  const bool in = b < whole * per_sample;
  const uint32_t j = in ? b >> 3 : b - whole * per_sample, s = j / per_sample;
  sample = in ? s * 8 + (b & 7) : whole + s;
  rest = j - s * per_sample;
}

// Forward.  APPLY: one part holds the sample (parts == 1) and the result is written; else only the part's mean and squared
// distances are left.  NP positions per lane.  Addresses are a uniform base and a 32-bit
// offset that walks, so that they cost two registers and not two per piece (with 64 registers of values that decides whether
// anything spills).  bf16 64 x 4096 x 256 in 32 groups with silu: 67 to 73 us, 3.7 to 4.0 TB/s where a copy moves 5.1: the vector units are
// busy 48 % of the time (18 instructions an element, two of them transcendental), which a workgroup as large as its CU's registers hides
// only in part.  In 512 lanes, two workgroups on a CU and 32 bytes of a position each, 99 us.
template <typename T, int V, int NP, bool APPLY, bool TAIL>
__global__ __launch_bounds__(1024) void norm_forward_kernel(NormArgs<T> a) {
  typedef Piece<T, V> Vec;
  __shared__ float red[2][16 * 64];
  const Place q = place_of<T, V, TAIL>(a);
  const uint32_t spb = blockDim.x / (uint32_t)a.D, per_sample = a.chunks * a.parts;
  for (uint32_t b = blockIdx.x; b < a.work; b += gridDim.x) {
    uint32_t si, rest;
    place_work(b, per_sample, a.work / per_sample, si, rest);
    const uint32_t chunk = rest % a.chunks, part = rest / a.chunks;
    const int64_t i0 = (int64_t)si * spb, i = i0 + q.sb;
    const int g = (int)chunk * a.gpc + q.g;
    const int pos0 = (int)part * a.PP, count_pos = (int)min((int64_t)a.PP, a.S - pos0);
    const bool live = i < a.n && g < a.G;
    const int count = live ? q.pieces(count_pos, a) : 0;               // of this lane
    const int64_t col0 = (int64_t)chunk * a.gpc * a.per;
    const char* const src = (const char*)(a.x + (i0 * a.S + pos0) * a.ldx + col0);
    const uint32_t lane_col = (uint32_t)(q.g * a.per + q.slot * V);
    Vec v[NP];
    {
      uint32_t off = ((uint32_t)(q.sb * (uint32_t)a.S + q.p) * (uint32_t)a.ldx + lane_col - (uint32_t)(V - q.nv)) * (uint32_t)sizeof(T);
      const uint32_t step = (uint32_t)a.PL * (uint32_t)a.ldx * (uint32_t)sizeof(T);
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        if (k < count) v[k].load(src + off);
        off += step;
        asm volatile("" : "+v"(off));
      }
    }
    const float elements = (float)count_pos * (float)a.per;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k)
      if (k < count) {
        if (TAIL) move_down(v[k], q.nv);
        float one = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) one += v[k].at(e);
        sum += one;
        v[k].hide();
      }
    const float mean = group_sum(sum, a.SP, a.TX, a.D, red[0]) / elements;
    float dist = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k)
      if (k < count) {
        float one = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) { const float d = v[k].at(e) - mean; one += TAIL && e >= q.nv ? 0.f : d * d; }
        dist += one;
        v[k].hide();
      }
    dist = group_sum(dist, a.SP, a.TX, a.D, red[1]);
    const bool first = live && q.p == 0 && q.slot == 0;
    if (!APPLY) {
      if (first) {
        float* o = a.part + ((i * a.G + g) * a.parts + part) * 2;
        o[0] = mean; o[1] = dist;
      }
    } else {
      const float rstd = rsqrtf(dist / elements + a.eps);
      if (first && a.mean) { a.mean[i * a.G + g] = mean; a.rstd[i * a.G + g] = rstd; }
      char* const dst = (char*)(a.y + (i0 * a.S + pos0) * a.ldy + col0);
      const uint32_t step = (uint32_t)a.PL * (uint32_t)a.ldy * (uint32_t)sizeof(T);
      if (count > 0) {
        float gam[V], bet[V];
        parameters<TAIL, T, V>(a, g * a.per + q.slot * V, q.nv, gam, bet);
#pragma unroll
        for (int e = 0; e < V; ++e) gam[e] *= rstd;
        uint32_t off = ((uint32_t)(q.sb * (uint32_t)a.S + q.p) * (uint32_t)a.ldy + lane_col) * (uint32_t)sizeof(T);
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          if (k < count) {
            float h[V];
            Vec o;
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = norm_h(v[k].at(e) - mean, gam[e], bet[e]);
            op_act_all<V, kFine<T>>(h, a.act);
            o.set(h);
            store_own<TAIL>(o, dst + off, q.nv);
          }
          off += step;
          asm volatile("" : "+v"(off));
        }
      }
    }
    // (red[0] is written again only behind the second sum's barrier, red[1] only behind the first one's)
  }
}

// Forward, single positions of wide groups: a workgroup per sample and group, kRow pieces along the channels in every lane, so that a lane
// has kRow loads under way and few wavefronts meet at the two sums.  bf16 4096 x 8192 in one group 27 us, 5.0 TB/s, the copy's rate (the
// kernel above, one piece a lane, 109), 4096 x 2048 9.8 (16), 16384 x 512 11.4 (14.6); 100 x 2000 6.5 (6.0).
constexpr int kRow = 4;
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = add_lanes<true>(v, 63);
  if (blockDim.x > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) v += red[w];
  }
  return v;
}
template <typename T, int V, bool TAIL>
__global__ __launch_bounds__(1024) void norm_row_kernel(NormArgs<T> a) {
  typedef Piece<T, V> Vec;
  __shared__ float red[2][16];
  const float inv = 1.0f / (float)a.per;
  for (uint32_t b = blockIdx.x; b < a.work; b += gridDim.x) {
    const uint32_t i = b / (uint32_t)a.G, g = b - i * (uint32_t)a.G;
    const int64_t c0 = (int64_t)g * a.per;
    const T* const src = a.x + i * a.ldx + c0;
    T* const dst = a.y + i * a.ldy + c0;
    auto slot_of = [&](int k) { return (int)threadIdx.x + k * (int)blockDim.x; };
    auto own = [&](int slot) { return TAIL ? min(V, a.per - slot * V) : V; };          // elements of a piece that are the group's
    Vec v[kRow];
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) v[k].load(src + (slot * V - (V - own(slot))));
    }
    float sum = 0.f, dist = 0.f;
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) {
        if (TAIL) move_down(v[k], own(slot));
#pragma unroll
        for (int e = 0; e < V; ++e) sum += v[k].at(e);
      }
    }
    const float mean = row_sum(sum, red[0]) * inv;
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) {
#pragma unroll
        for (int e = 0; e < V; ++e) { const float d = v[k].at(e) - mean; dist += TAIL && e >= own(slot) ? 0.f : d * d; }
      }
    }
    const float rstd = rsqrtf(row_sum(dist, red[1]) * inv + a.eps);
    if (threadIdx.x == 0 && a.mean) { a.mean[b] = mean; a.rstd[b] = rstd; }
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) {
        float gam[V], bet[V], h[V];
        parameters<TAIL, T, V>(a, (int)c0 + slot * V, own(slot), gam, bet);
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = norm_h(v[k].at(e) - mean, gam[e] * rstd, bet[e]);
        op_act_all<V, kFine<T>>(h, a.act);
        Vec o;
        o.set(h);
        store_own<TAIL>(o, dst + slot * V, own(slot));
      }
    }
    // (red[0] is written again only behind the second sum's barrier, red[1] only behind the first one's)
  }
}

// Joins the parts' statistics and writes; a workgroup takes the positions of one part.
template <typename T, int V, bool TAIL>
__global__ __launch_bounds__(1024) void norm_apply_kernel(NormArgs<T> a) {
  typedef Piece<T, V> Vec;
  const Place q = place_of<T, V, TAIL>(a);
  for (uint32_t b = blockIdx.x; b < a.work; b += gridDim.x) {
    const uint32_t chunk = b % a.chunks, part = b / a.chunks % a.parts;
    const int64_t i = b / a.chunks / a.parts;
    const int g = (int)chunk * a.gpc + q.g;
    if (g >= a.G || q.slot >= a.slots) continue;
    const float2* st = (const float2*)a.part + (i * a.G + g) * a.parts;
    float mean = 0.f, dist = 0.f;
    const float inv = 1.0f / ((float)a.S * (float)a.per), full = (float)a.PP * (float)a.per;
    const uint32_t last = a.parts - 1;
    const float rest = (float)(a.S - (int64_t)last * a.PP) * (float)a.per;
#pragma unroll 8
    for (uint32_t k = 0; k < a.parts; ++k) mean += st[k].x * ((k < last ? full : rest) * inv);
#pragma unroll 8
    for (uint32_t k = 0; k < a.parts; ++k) {
      const float d = st[k].x - mean;
      dist += fmaf((k < last ? full : rest) * d, d, st[k].y);
    }
    const float rstd = rsqrtf(dist * inv + a.eps);
    if (a.mean && part == 0 && q.p == 0 && q.slot == 0) { a.mean[i * a.G + g] = mean; a.rstd[i * a.G + g] = rstd; }
    float gam[V], bet[V];
    parameters<TAIL, T, V>(a, g * a.per + q.slot * V, q.nv, gam, bet);
#pragma unroll
    for (int e = 0; e < V; ++e) gam[e] *= rstd;
    const int pos0 = (int)part * a.PP, count_pos = (int)min((int64_t)a.PP, a.S - pos0);
    const int64_t col = (int64_t)g * a.per + q.slot * V;
    const T* src = a.x + (i * a.S + pos0 + q.p) * a.ldx + col;
    T* dst = a.y + (i * a.S + pos0 + q.p) * a.ldy + col;
#pragma unroll 4
    for (int pos = q.p; pos < count_pos; pos += a.PL) {
      Vec v, o;
      load_own<TAIL>(v, src, q.nv);
      float h[V];
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = norm_h(v.at(e) - mean, gam[e], bet[e]);
      op_act_all<V, kFine<T>>(h, a.act);
      o.set(h);
      store_own<TAIL>(o, dst, q.nv);
      src += a.PL * a.ldx;
      dst += a.PL * a.ldy;
    }
  }
}

// dh of one piece, and the distances d from the mean.  s: gamma rstd
template <typename T, int V>
__device__ __forceinline__ void norm_dh(const Piece<T, V>& x, const Piece<T, V>& dy, float mean, const float* s, const float* bet, int act,
                                        float* d, float* dh) {
  float h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    d[e] = x.at(e) - mean;
    dh[e] = dy.at(e);
  }
  if (act != ABS_ACT_NONE) {
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = norm_h(d[e], s[e], bet[e]);
    op_slope_all<V, kFine<T>>(dh, h, act);
  }
}

// Backward.  A workgroup keeps its chunk of channels for all its samples, so that the shares of dgamma and dbeta add up in
// registers and leave once per workgroup.  APPLY as in the forward pass: else only the parts' two sums (and the shares).
// dh stays in fp32 registers between the sums and dx.  What is added per element are dh and dh d alone, per channel of the lane's piece:
// with s = gamma rstd the group's two sums are S1 = sum_c s_c sum dh and S2 = sum_c s_c sum (dh d), a channel's share of dgamma is
// rstd sum (dh d), and dx = s dh - S1 / N - d rstd^2 S2 / N.  bf16 with silu: 32 x 1024 x 512 in 32 groups 37 us + 5 for the shares,
// 8192 x 2048 with residual 38 + 5; the bytes alone 17 and 22.  The vector units are busy 41 and 51 % of the time (41 and 48 instructions an element),
// a wavefront waits 43 and 46 % of its: loads, sums and stores of a share come one after the other (two workgroups on a CU, and with single
// positions the next share's loads, cover some of it), and a workgroup of the first asks for 32 bytes of a position, a quarter of a line.
template <typename T, int V, int NP, bool APPLY, bool TAIL>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormArgs<T> a) {
  typedef Piece<T, V> Vec;
  constexpr bool kKeep = APPLY && NP * V <= 32;
  constexpr bool kLean = NP * V >= 32;            // no registers for what only the next share needs: sums in LDS, parameters read again
  __shared__ float red[2][16 * 64];
  extern __shared__ float share[];
  const Place q = place_of<T, V, TAIL>(a);
  const uint32_t spb = blockDim.x / (uint32_t)a.D;
  uint32_t chunk, row;
  place_work(blockIdx.x, a.chunks, a.row_count, row, chunk);
  const int g = (int)chunk * a.gpc + q.g;
  float gam[V], bet[V], sg[V], sb[V];
  auto channels = [&]() {
    int s = q.slot;
    asm volatile("" : "+v"(s));
#pragma unroll
    for (int e = 0; e < V; ++e) { gam[e] = 1.f; bet[e] = 0.f; }
    if (g < a.G && s < a.slots) parameters<TAIL, T, V>(a, g * a.per + s * V, q.nv, gam, bet);
  };
  if (!kLean) {
    channels();
#pragma unroll
    for (int e = 0; e < V; ++e) sg[e] = sb[e] = 0.f;
  }
  const uint32_t work = a.work / a.chunks;
  const float inv = 1.0f / ((float)a.S * (float)a.per);
  const int64_t col0 = (int64_t)chunk * a.gpc * a.per;
  const uint32_t lane_col = (uint32_t)(q.g * a.per + q.slot * V), lane_pos = (uint32_t)(q.sb * (uint32_t)a.S + q.p);
  // a lane's first piece in each array, as 32-bit offsets from the workgroup's place there
  auto offset = [&](int64_t ld) { return (lane_pos * (uint32_t)ld + lane_col) * (uint32_t)sizeof(T); };
  uint32_t ox0, od0, or0, oy0;
  if (!kLean) { ox0 = offset(a.ldx); od0 = offset(a.lddy); or0 = offset(a.lddres); oy0 = offset(a.ldy); }
  auto first = [&](uint32_t kept, int64_t ld) {
    if (!kLean) return kept;
    uint32_t pos = lane_pos;
    asm volatile("" : "+v"(pos));
    return (pos * (uint32_t)ld + lane_col) * (uint32_t)sizeof(T);
  };
  auto walk = [&](uint32_t& off, int64_t ld) {
    off += (uint32_t)a.PL * (uint32_t)ld * (uint32_t)sizeof(T);
    asm volatile("" : "+v"(off));
  };
  // What a workgroup's next share needs is asked for before this one's is worked on, where that is few registers: with single
  // positions a share is over in the time of a load.
  constexpr bool kAhead = NP * Vec::kWords <= 4;
  struct Fetched { Vec x[NP], dy[NP], res[kAhead ? NP : 1]; float mean, rstd; int count; int64_t stat; uint32_t part; };
  // Uniform places of the share to be fetched: samples a.row_count shares on, or parts of them.
  const int64_t base = col0 * (int64_t)sizeof(T);
  struct Spot { const char *x, *dy, *res; char* y; int64_t i0; };
  auto spot_of = [&](uint32_t b) {
    const uint32_t s = a.parts == 1 ? b : b / a.parts;
    const int64_t i0 = (int64_t)s * spb, at = i0 * a.S + (int64_t)(b - s * a.parts) * a.PP;
    return Spot{(const char*)a.x + at * a.ldx * (int64_t)sizeof(T) + base, (const char*)a.dy + at * a.lddy * (int64_t)sizeof(T) + base,
                (const char*)a.dres + at * a.lddres * (int64_t)sizeof(T) + base, (char*)a.y + at * a.ldy * (int64_t)sizeof(T) + base, i0};
  };
  const int64_t hop = (int64_t)a.row_count * spb;                       // parts == 1: samples between a workgroup's shares
  const int64_t hop_bytes = hop * a.S * (int64_t)sizeof(T);
  auto fetch = [&](uint32_t b, const Spot& p, Fetched& f) {
    f.part = a.parts == 1 ? 0u : b % a.parts;
    const int64_t i = p.i0 + q.sb;
    const bool live = i < a.n && g < a.G;
    f.count = live ? q.pieces((int)min((int64_t)a.PP, a.S - (int64_t)f.part * a.PP), a) : 0;
    uint32_t ox = first(ox0, a.ldx), od = first(od0, a.lddy), orr = kAhead ? first(or0, a.lddres) : 0;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      if (k < f.count) {
        const uint32_t early = TAIL ? (uint32_t)(V - q.nv) * (uint32_t)sizeof(T) : 0;
        f.x[k].load(p.x + (ox - early));
        f.dy[k].load(p.dy + (od - early));
        if (APPLY && kAhead && a.dres) load_own<TAIL>(f.res[kAhead ? k : 0], p.res + orr, q.nv);
      }
      if (NP > 1) { walk(ox, a.ldx); walk(od, a.lddy); if (kAhead) walk(orr, a.lddres); }
    }
    f.stat = i * a.G + g;
    f.mean = live ? a.mean[f.stat] : 0.f;
    f.rstd = live ? a.rstd[f.stat] : 0.f;
  };
  Fetched next;
  Spot here = spot_of(row), there = here;
  if (kAhead && row < work) fetch(row, here, next);
  for (uint32_t b = row; b < work; b += a.row_count) {
    Fetched now;
    if (a.parts > 1) { if (b != row) here = spot_of(b); }
    else if (b != row) here = there;
    if (kAhead && a.parts > 1) there = spot_of(b + a.row_count);
    else there = Spot{here.x + hop_bytes * a.ldx, here.dy + hop_bytes * a.lddy, here.res + hop_bytes * a.lddres, here.y + hop_bytes * a.ldy, here.i0 + hop};
    if (kAhead) { now = next; if (b + a.row_count < work) fetch(b + a.row_count, there, next); }
    else fetch(b, here, now);
    Vec* const vx = now.x;
    Vec* const vd = now.dy;
    const float mean = now.mean, rstd = now.rstd;
    const int count = now.count;
    if (kLean) channels();
    float kept[kKeep ? NP * V : 1], s[V], lb[V], lg[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { s[e] = gam[e] * rstd; lb[e] = lg[e] = 0.f; }
#pragma unroll
    for (int k = 0; k < NP; ++k)
      if (k < count) {
        if (TAIL) { move_down(vx[k], q.nv); move_down(vd[k], q.nv); }
        float d[V], dh[V];
        norm_dh<T, V>(vx[k], vd[k], mean, s, bet, a.act, d, dh);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          lb[e] += dh[e];
          lg[e] = fmaf(dh[e], d[e], lg[e]);
          if (kKeep) kept[k * V + e] = dh[e];
        }
        vx[k].hide();
        if (!kKeep) vd[k].hide();
      }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      s1 = fmaf(s[e], lb[e], s1);
      s2 = fmaf(s[e], lg[e], s2);
      if (!kLean) {
        sb[e] += lb[e];
        sg[e] = fmaf(rstd, lg[e], sg[e]);
      }
    }
    if (kLean) {                                    // a lane's own place, first written and then added to
      uint32_t at = threadIdx.x * (2 * V);
      asm volatile("" : "+v"(at));
      float* const own = share + at;
#pragma unroll
      for (int e = 0; e < V; ++e) { sg[e] = sb[e] = 0.f; }
      if (b != row) {
#pragma unroll
        for (int e = 0; e < V; ++e) { sg[e] = own[e]; sb[e] = own[V + e]; }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) { own[e] = fmaf(rstd, lg[e], sg[e]); own[V + e] = lb[e] + sb[e]; }
    }
    s1 = group_sum(s1, a.SP, a.TX, a.D, red[0]);
    s2 = group_sum(s2, a.SP, a.TX, a.D, red[1]);
    if (!APPLY) {
      if (count > 0 && q.p == 0 && q.slot == 0) {
        float* o = a.part + (now.stat * a.parts + now.part) * 2;
        o[0] = s1; o[1] = s2;
      }
    } else {
      const float c1 = -(s1 * inv), c2 = -rstd * (rstd * (s2 * inv));
      uint32_t oy = first(oy0, a.ldy), orr = a.dres ? first(or0, a.lddres) : 0;
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        if (k < count) {
          float d[V], w[V];
          if constexpr (kKeep) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              d[e] = vx[k].at(e) - mean;
              w[e] = kept[k * V + e];
            }
          } else {
            norm_dh<T, V>(vx[k], vd[k], mean, s, bet, a.act, d, w);
          }
          Vec o, r;
          if (a.dres) { if constexpr (kAhead) r = now.res[k]; else load_own<TAIL>(r, here.res + orr, q.nv); }
#pragma unroll
          for (int e = 0; e < V; ++e) {
            w[e] = fmaf(s[e], w[e], fmaf(c2, d[e], c1));
            if (a.dres) w[e] += r.at(e);
          }
          o.set(w);
          store_own<TAIL>(o, here.y + oy, q.nv);
        }
        if (NP > 1) { walk(oy, a.ldy); walk(orr, a.lddres); }
      }
    }
  }
  if (!a.rows_g) return;
  if (kLean) {
#pragma unroll
    for (int e = 0; e < V; ++e) { sg[e] = share[threadIdx.x * (2 * V) + e]; sb[e] = share[threadIdx.x * (2 * V) + V + e]; }
    __syncthreads();
  }
  // the lanes that share a channel: positions and samples of the workgroup
  const int t = threadIdx.x, lanes = min(a.TX, 64), stack = blockDim.x / (a.TX > 64 ? a.TX : 64);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    sg[e] = add_lanes<false>(sg[e], 63 & ~(a.TX - 1));
    sb[e] = add_lanes<false>(sb[e], 63 & ~(a.TX - 1));
  }
  if (stack > 1) {                                // [stack][V][TX], dgamma's shares and then dbeta's
    const int r = t / (a.TX > 64 ? a.TX : 64), tx = t & (a.TX - 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h) __syncthreads();
      if (a.TX >= 64 || (t & 63) < lanes) {
#pragma unroll
        for (int e = 0; e < V; ++e) share[(r * V + e) * a.TX + tx] = h ? sb[e] : sg[e];
      }
      __syncthreads();
      if (t < a.TX) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float sum = 0.f;
          for (int k = 0; k < stack; ++k) sum += share[(k * V + e) * a.TX + t];
          (h ? sb : sg)[e] = sum;
        }
      }
    }
  }
  if (t >= a.TX) return;
  if (g < a.G && q.slot < a.slots) {
    const int64_t o = (int64_t)row * a.row_step + (int64_t)g * a.per + q.slot * V;
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < q.nv) { a.rows_g[o + e] = sg[e]; a.rows_b[o + e] = sb[e]; }
  }
}

template <typename T, int V, bool TAIL>
__global__ __launch_bounds__(1024) void norm_backward_apply_kernel(NormArgs<T> a) {
  typedef Piece<T, V> Vec;
  const Place q = place_of<T, V, TAIL>(a);
  const float inv = 1.0f / ((float)a.S * (float)a.per);
  for (uint32_t b = blockIdx.x; b < a.work; b += gridDim.x) {
    const uint32_t chunk = b % a.chunks, part = b / a.chunks % a.parts;
    const int64_t i = b / a.chunks / a.parts;
    const int g = (int)chunk * a.gpc + q.g;
    if (g >= a.G || q.slot >= a.slots) continue;
    const float2* st = (const float2*)a.part + (i * a.G + g) * a.parts;
    float m1 = 0.f, m2 = 0.f;
#pragma unroll 8
    for (uint32_t k = 0; k < a.parts; ++k) { m1 += st[k].x; m2 += st[k].y; }
    const float mean = a.mean[i * a.G + g], rstd = a.rstd[i * a.G + g];
    const float c1 = -(m1 * inv), c2 = -rstd * (rstd * (m2 * inv));
    float sc[V], bet[V];
    parameters<TAIL, T, V>(a, g * a.per + q.slot * V, q.nv, sc, bet);
#pragma unroll
    for (int e = 0; e < V; ++e) sc[e] *= rstd;
    const int pos0 = (int)part * a.PP, count_pos = (int)min((int64_t)a.PP, a.S - pos0);
    const int64_t at = i * a.S + pos0 + q.p, col = (int64_t)g * a.per + q.slot * V;
    const T* px = a.x + at * a.ldx + col;
    const T* pd = a.dy + at * a.lddy + col;
    const T* pr = a.dres ? a.dres + at * a.lddres + col : nullptr;
    T* dst = a.y + at * a.ldy + col;
    const int early = TAIL ? V - q.nv : 0;                    // (dx may be dres, never x or dy)
#pragma unroll 4
    for (int pos = q.p; pos < count_pos; pos += a.PL) {
      Vec vx, vd, o, r;
      vx.load(px - early); vd.load(pd - early);
      if (pr) load_own<TAIL>(r, pr, q.nv);
      if (TAIL) { move_down(vx, q.nv); move_down(vd, q.nv); }
      float d[V], dh[V];
      norm_dh<T, V>(vx, vd, mean, sc, bet, a.act, d, dh);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        dh[e] = fmaf(sc[e], dh[e], fmaf(c2, d[e], c1));
        if (pr) dh[e] += r.at(e);
      }
      o.set(dh);
      store_own<TAIL>(o, dst, q.nv);
      px += a.PL * a.ldx; pd += a.PL * a.lddy; dst += a.PL * a.ldy;
      if (pr) pr += a.PL * a.lddres;
    }
  }
}

// Backward, single positions of wide groups, like norm_row_kernel: a workgroup takes every row_count-th sample of one group, so that its
// channels' sums add up in registers.  gamma and beta are read again for every sample (they are in the caches).  Groups of whole pieces
// alone: the registers do not hold a partial piece's handling too (4096 x 4099 fp32 125 -> 139 us).  4096 x 8192 bf16 in one group 61 us
// (79 in norm_backward_kernel, floor 39), x 16384 127 (366 in the plain kernel, floor 78), fp32 4096 x 4096 51 (130); 4096 x 2048
// bf16 34 against 30 there, hence the rule.
template <typename T, int V>
__global__ __launch_bounds__(1024) void norm_row_backward_kernel(NormArgs<T> a) {
  typedef Piece<T, V> Vec;
  __shared__ float red[2][16];
  const float inv = 1.0f / (float)a.per;
  const uint32_t row = blockIdx.x / (uint32_t)a.G, g = blockIdx.x - row * (uint32_t)a.G;
  const int c0 = (int)g * a.per;
  auto slot_of = [&](int k) { return (int)threadIdx.x + k * (int)blockDim.x; };
  float sg[kRow][V], sb[kRow][V];
#pragma unroll
  for (int k = 0; k < kRow; ++k)
#pragma unroll
    for (int e = 0; e < V; ++e) sg[k][e] = sb[k][e] = 0.f;
  for (int64_t i = row; i < a.n; i += a.row_count) {
    const T* const px = a.x + i * a.ldx + c0;
    const T* const pd = a.dy + i * a.lddy + c0;
    Vec x[kRow], dy[kRow];
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) {
        x[k].load(px + slot * V);
        dy[k].load(pd + slot * V);
      }
    }
    const float mean = a.mean[i * a.G + g], rstd = a.rstd[i * a.G + g];
    float kept[kRow][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) {
        float s[V], bet[V], d[V], dh[V];
        parameters<false, T, V>(a, c0 + slot * V, V, s, bet);
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] *= rstd;
        norm_dh<T, V>(x[k], dy[k], mean, s, bet, a.act, d, dh);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sb[k][e] += dh[e];
          sg[k][e] = fmaf(rstd, dh[e] * d[e], sg[k][e]);
          kept[k][e] = s[e] * dh[e];
          s1 += kept[k][e];
          s2 = fmaf(kept[k][e], d[e], s2);
        }
        x[k].hide();
      }
    }
    s1 = row_sum(s1, red[0]);
    s2 = row_sum(s2, red[1]);
    const float c1 = -(s1 * inv), c2 = -rstd * (rstd * (s2 * inv));
    T* const py = a.y + i * a.ldy + c0;
    const T* const pr = a.dres ? a.dres + i * a.lddres + c0 : nullptr;
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
      const int slot = slot_of(k);
      if (slot < a.slots) {
        Vec o, res;
        if (pr) res.load(pr + slot * V);
        float w[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          w[e] = kept[k][e] + fmaf(c2, x[k].at(e) - mean, c1);
          if (pr) w[e] += res.at(e);
        }
        o.set(w);
        o.store(py + slot * V);
      }
    }
    // (red[0] is written again only behind the second sum's barrier, red[1] only behind the first one's)
  }
  if (!a.rows_g) return;
#pragma unroll
  for (int k = 0; k < kRow; ++k) {
    const int slot = slot_of(k);
    if (slot < a.slots) {
      const int64_t o = (int64_t)row * a.row_step + c0 + slot * V;
#pragma unroll
      for (int e = 0; e < V; ++e) { a.rows_g[o + e] = sg[k][e]; a.rows_b[o + e] = sb[k][e]; }
    }
  }
}

// dgamma, dbeta: the workgroups' shares added in their order, 32 channels x 32 rows of shares at a time, eight rows of a lane in
// flight (423 shares of 69 channels 16 -> 6 us)
__global__ __launch_bounds__(1024) void norm_share_sum_kernel(const float* rows, uint32_t row_count, int C, float* dgamma, float* dbeta) {
  __shared__ float s[32][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  const float* p = rows + (blockIdx.y ? C : 0) + c;
  float v = 0.f;
  if (c < C)
#pragma unroll 8
    for (uint32_t k = r; k < row_count; k += 32) v += p[(int64_t)k * 2 * C];
  s[r][threadIdx.x & 31] = v;
  __syncthreads();
  if (r == 0 && c < C) {
    v = 0.f;
    for (int k = 0; k < 32; ++k) v += s[k][threadIdx.x];
    (blockIdx.y ? dbeta : dgamma)[c] = v;
  }
}

// ---- groups of any width: a workgroup per sample and group, every pass over memory (bf16 64 x 65536 in one group 50 us, gradient 89,
// the bytes alone 3 and 5) ---------------------
__device__ __forceinline__ float block_sum(float v, float* red) {
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) v += red[w];
  return v;
}

template <typename T, bool BACKWARD>
__global__ __launch_bounds__(1024) void norm_plain_kernel(NormArgs<T> a) {
  __shared__ float red[16];
  const float inv = 1.0f / ((float)a.S * (float)a.per);
  for (int64_t b = blockIdx.x; b < a.n * a.G; b += gridDim.x) {
    const int64_t i = b / a.G;
    const int g = (int)(b % a.G), c0 = g * a.per;
    float mean, rstd, m1 = 0.f, m2 = 0.f;
    if (!BACKWARD) {
      float sum = 0.f;
      for (int64_t pos = 0; pos < a.S; ++pos)
        for (int c = threadIdx.x; c < a.per; c += blockDim.x) sum += op_widen(a.x[(i * a.S + pos) * a.ldx + c0 + c]);
      mean = block_sum(sum, red) * inv;
      float dist = 0.f;
      for (int64_t pos = 0; pos < a.S; ++pos)
        for (int c = threadIdx.x; c < a.per; c += blockDim.x) {
          const float d = op_widen(a.x[(i * a.S + pos) * a.ldx + c0 + c]) - mean;
          dist += d * d;
        }
      rstd = rsqrtf(block_sum(dist, red) * inv + a.eps);
      if (threadIdx.x == 0 && a.mean) { a.mean[b] = mean; a.rstd[b] = rstd; }
    } else {
      mean = a.mean[b]; rstd = a.rstd[b];
      float s1 = 0.f, s2 = 0.f;
      for (int64_t pos = 0; pos < a.S; ++pos)
        for (int c = threadIdx.x; c < a.per; c += blockDim.x) {
          const float gam = a.gamma ? a.gamma[c0 + c] : 1.f, bet = a.gamma ? a.beta[c0 + c] : 0.f;
          const float d = op_widen(a.x[(i * a.S + pos) * a.ldx + c0 + c]) - mean, s = gam * rstd;
          const float w = op_slope<kFine<T>>(op_widen(a.dy[(i * a.S + pos) * a.lddy + c0 + c]), norm_h(d, s, bet), a.act) * s;
          s1 += w; s2 += w * d;
        }
      m1 = block_sum(s1, red) * inv;
      m2 = rstd * (rstd * (block_sum(s2, red) * inv));
    }
    for (int64_t pos = 0; pos < a.S; ++pos)
      for (int c = threadIdx.x; c < a.per; c += blockDim.x) {
        const int64_t at = i * a.S + pos;
        const float gam = a.gamma ? a.gamma[c0 + c] : 1.f, bet = a.gamma ? a.beta[c0 + c] : 0.f;
        const float d = op_widen(a.x[at * a.ldx + c0 + c]) - mean, s = gam * rstd, h = norm_h(d, s, bet);
        float v;
        if (!BACKWARD) v = op_act<kFine<T>>(h, a.act);
        else {
          v = op_slope<kFine<T>>(op_widen(a.dy[at * a.lddy + c0 + c]), h, a.act) * s - m1 - d * m2;
          if (a.dres) v += op_widen(a.dres[at * a.lddres + c0 + c]);
        }
        op_narrow(v, a.y[at * a.ldy + c0 + c]);
      }
  }
}

// ... and their shares of dgamma, dbeta: a thread per channel, row_count runs of positions.  Stands before norm_plain_kernel, which
// may write dx over dres but never over x or dy.
template <typename T>
__global__ __launch_bounds__(256) void norm_plain_share_kernel(NormArgs<T> a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.C) return;
  const int g = (int)c / a.per;
  const float gam = a.gamma ? a.gamma[c] : 1.f, bet = a.gamma ? a.beta[c] : 0.f;
  const int64_t total = a.n * a.S;
  for (uint32_t r = blockIdx.y; r < a.row_count; r += gridDim.y) {
    float sg = 0.f, sb = 0.f;
    for (int64_t at = r; at < total; at += a.row_count) {
      const int64_t i = at / a.S;
      const float d = op_widen(a.x[at * a.ldx + c]) - a.mean[i * a.G + g], rstd = a.rstd[i * a.G + g];
      const float dh = op_slope<kFine<T>>(op_widen(a.dy[at * a.lddy + c]), norm_h(d, gam * rstd, bet), a.act);
      sg += dh * (d * rstd); sb += dh;
    }
    a.rows_g[(int64_t)r * a.row_step + c] = sg;
    a.rows_b[(int64_t)r * a.row_step + c] = sb;
  }
}

// ---- the plan -------------------------------------------------------------------------------------------
struct NormPlan {
  int V, NP, threads;
  bool tail, plain, split, row;
  int slots, SP, gpc, TX, PL, D, PP;
  uint32_t chunks, parts, row_count, work, blocks;
  size_t off_rows, bytes;                  // workspace: parts' statistics, then the shares of dgamma / dbeta
};

int pow2_up(int64_t x) { int p = 1; while (p < x) p <<= 1; return p; }

// Single positions of groups so wide that several pieces a lane pay: norm_row_kernel, norm_row_backward_kernel.
bool norm_rows(const abs_group_norm& p, bool backward, int V) {
  const int per = p.channels / p.groups, slots = (per + V - 1) / V;
  return p.spatial == 1 && slots <= kRow * 1024 && p.n * p.groups < 1ll << 31 && (backward ? V == 4 && per % 4 == 0 && per >= 4096 : slots > 32);
}

// The widest piece: 16 bytes; backward four elements, but for single positions (norm_piece).
int norm_widest(const abs_group_norm& p, bool backward) { return p.dtype == ABS_X_BF16 && (!backward || (p.spatial == 1 && !norm_rows(p, true, 4))) ? 8 : 4; }

// V: elements of a piece.
NormPlan norm_plan(const abs_group_norm& p, bool backward, int V) {
  NormPlan q{};
  const int size = op_size(p.dtype), per = p.channels / p.groups;
  const int64_t S = p.spatial;
  q.V = V; q.tail = per % V != 0; q.parts = 1; q.PP = (int)S;
  q.slots = (per + V - 1) / V;
  q.SP = pow2_up(q.slots);
  const int np_most = backward ? 8 : 16;
  if (norm_rows(p, backward, V)) {
    q.row = true;
    q.threads = std::max(64, pow2_up((q.slots + kRow - 1) / kRow));
    q.work = (uint32_t)(p.n * p.groups);
    q.blocks = std::min(q.work, 1u << 20);
    if (backward) {
      q.row_count = (uint32_t)std::min<int64_t>(p.n, std::max(1, 256 * (1024 / q.threads) / p.groups));
      q.blocks = q.row_count * (uint32_t)p.groups;
      if (q.row_count > 1) q.bytes = op_round_up((size_t)q.row_count * 2 * p.channels * 4, 256);
    }
    return q;
  }
  if (q.SP > kMaxLanes) {
    q.plain = true;
  } else {
    // groups side by side: 128 bytes of a position, more while a sample has less than a wavefront's pieces
    const int g_most = std::min(pow2_up(p.groups), kMaxLanes / q.SP);
    q.gpc = 1;
    while (q.gpc < g_most && ((int64_t)q.gpc * per * size < 128 || q.gpc * q.SP * S < 256)) q.gpc *= 2;
    // ... fewer, down to 32 bytes, where only that lets a workgroup hold a sample
    // (backward: half of its lanes where that does it: two workgroups share a CU, and one loads while the other works)
    auto lanes = [&](int gpc) { return (int64_t)gpc * q.SP * pow2_up((S + np_most - 1) / np_most); };
    auto narrow = [&](int most) {
      int gpc = q.gpc;
      while (gpc > 1 && lanes(gpc) > most && (int64_t)(gpc / 2) * per * size >= 32) gpc /= 2;
      if (lanes(gpc) > most) return false;
      q.gpc = gpc;
      return true;
    };
    q.split = !(backward && narrow(kMaxLanes / 2)) && !narrow(kMaxLanes);
    q.TX = q.gpc * q.SP;
    q.chunks = (p.groups + q.gpc - 1) / q.gpc;
    // few workgroups with much to do each: parts as well
    if (!q.split && p.n * q.chunks < 128 && S * q.TX >= 4096) q.split = true;
    if (q.split) {
      const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(1, p.n * q.chunks));       // parts that fill the chip
      const int pl = std::max(1, std::min(kMaxLanes, std::max(256, q.TX)) / q.TX);
      int64_t pp = (S + want - 1) / want;
      const int most = pl * np_most;
      pp = std::max<int64_t>(pp, (1024 + q.TX - 1) / q.TX);         // (16 KB of 16-byte pieces)
      if (pp > most) pp = most;
      q.NP = pp <= pl ? 1 : pp <= 4 * pl ? 4 : np_most;
      q.PL = pow2_up((pp + q.NP - 1) / q.NP);
      q.PP = q.PL * q.NP;
      q.parts = (uint32_t)((S + q.PP - 1) / q.PP);
      q.D = q.TX * q.PL;
    } else {
      // As few positions a lane as half a workgroup takes while the lanes are few, more where more positions leave lanes enough: what a
      // lane does once - its place, the sums across lanes - takes the time of several pieces (bf16 6140 x 9 x 224 in 32 groups 85 -> 21 us,
      // gradient 88 -> 41; 500 x 9 x 224 10.7 -> 6.4, 16.8 -> 13; 4000 x 49 x 64 in 8 34 -> 15; 100000 x 4 x 64 35 -> 24, but its
      // gradient 58 -> 62).
      q.NP = np_most;
      auto lanes_at = [&](int np) { return (int64_t)q.TX * pow2_up((S + np - 1) / np); };
      for (int np : {1, 4, np_most}) {
        const int more = np == 1 ? 4 : backward && size == 4 ? 0 : np_most;       // (eight positions of fp32 spill in the backward pass)
        if (lanes_at(np) <= 512 && (np == np_most || S <= np || !more || p.n * q.chunks * lanes_at(more) < kPlenty)) { q.NP = np; break; }
      }
      q.PL = pow2_up((S + q.NP - 1) / q.NP);
      q.D = q.TX * q.PL;
    }
  }
  size_t o = 0;
  if (!q.plain) {
    // a workgroup's samples lie within 32-bit offsets of its first one
    q.threads = q.split ? q.D : std::max(q.D, 256);
    // (backward: the more samples share a workgroup, the fewer shares of dgamma and dbeta)
    if (backward && !q.split)
      while (q.threads < 512 && p.n * q.D / (2 * q.threads) * q.chunks >= 512) q.threads *= 2;
    const int64_t spb = q.threads / q.D, reach = spb * S;
    const int64_t ld = std::max({p.ldx, backward ? p.lddy : p.ldy, backward ? p.lddx : 0, backward ? p.lddres : 0});
    const int64_t work = (p.n + spb - 1) / spb * q.parts * q.chunks;
    if ((double)reach * (double)ld * size >= 4.0e9 || work >= 1ll << 31) { q.plain = true; q.split = false; q.parts = 1; }
    else q.work = (uint32_t)work;
  }
  if (q.plain) {
    q.threads = 1024;
    q.blocks = (uint32_t)std::min<int64_t>(p.n * p.groups, 4096);
    q.row_count = (uint32_t)std::min<int64_t>(64, p.n * S);
  } else {
    if (backward) {
      // as many workgroups as the CUs hold at once (1024 lanes each by their registers); a workgroup per share where a share has
      // so many positions that its two numbers per channel do not count
      const uint32_t fill = std::max(1u, 256u * (1024u / (uint32_t)q.threads) / q.chunks), all = q.work / q.chunks;
      const bool fits = (int64_t)all * q.chunks * q.threads < 1ll << 32;                              // (a launch's threads)
      q.row_count = (int64_t)q.threads / q.D * q.PL * q.NP >= 64 && all <= 4096 && fits ? all : std::min(all, fill);
      // little work is one workgroup's per chunk: its sums are dgamma and dbeta, and the launch that adds shares is spared
      if (!q.split && all <= 4 && (all - 1) * q.NP <= 8) q.row_count = 1;
      q.blocks = q.row_count * q.chunks;
    } else {
      q.blocks = std::min(q.work, 1u << 20);
    }
    if (q.split) o = op_round_up((size_t)p.n * p.groups * q.parts * 8, 256);
  }
  q.off_rows = o;
  if (backward && q.row_count > 1) o += op_round_up((size_t)q.row_count * 2 * p.channels * 4, 256);
  q.bytes = o;
  return q;
}

// A piece's elements, at any pitch and alignment: as many as fit, where a group is a whole number of them; other groups end in a
// piece that is partly theirs, of four elements (two for groups of two and three).  Backward eight only for single positions: the sums and
// parameters of a piece's channels fill the registers that more positions need.  (bf16 gradients, four and a part against single elements:
// 47 x 2116 x 69 in one group 51 and 103 us, 1622 x 289 x 10 in two 47 and 79; eight against four: 8192 x 2048 in 32 groups 44 and 47.)
int norm_piece(const abs_group_norm& p, bool backward) {
  const int per = p.channels / p.groups, most = norm_widest(p, backward);
  return per % most == 0 ? most : per >= 4 ? 4 : per >= 2 ? 2 : 1;
}

const char* norm_problem(const abs_group_norm* p, bool backward) {
  if (!p) return "group norm: the description is NULL";
  if (p->dtype != ABS_X_FP32 && p->dtype != ABS_X_BF16) return "group norm: dtype must be ABS_X_FP32 or ABS_X_BF16";
  if (p->act < ABS_ACT_NONE || p->act > ABS_ACT_GELU) return "group norm: act must be 0..3";
  if (p->reserved != 0) return "group norm: reserved must be 0";
  if (p->n < 0 || p->spatial < 1 || p->spatial > 0x7FFFFFFF || p->n > 0x7FFFFFFF || p->n * p->spatial > 0x7FFFFFFF)
    return "group norm: n >= 0, spatial >= 1 and n x spatial < 2^31";
  if (p->channels < 1 || p->channels > 1 << 20) return "group norm: channels must be in [1, 2^20]";
  if (p->groups < 1 || p->groups > p->channels || p->channels % p->groups) return "group norm: groups must divide channels";
  if (!(p->eps >= 0.f) || p->eps > 1e30f) return "group norm: eps must be finite and not negative";
  if (p->ldx < p->channels || (backward ? p->lddy < p->channels || p->lddx < p->channels : p->ldy < p->channels))
    return "group norm: a pitch is below channels";
  constexpr int64_t most = 1ll << 40;
  if (p->ldx >= most || (backward ? p->lddy >= most || p->lddx >= most : p->ldy >= most)) return "group norm: a pitch is 2^40 or more";
  return nullptr;
}

template <typename T>
void norm_fill(NormArgs<T>& a, const abs_group_norm& p, const NormPlan& q, char* ws) {
  a.n = p.n; a.S = p.spatial; a.C = p.channels; a.G = p.groups; a.per = p.channels / p.groups; a.act = p.act; a.eps = p.eps;
  a.ldx = p.ldx;
  a.slots = q.slots; a.SP = q.SP; a.gpc = q.gpc; a.TX = q.TX; a.PL = q.PL; a.D = q.D; a.chunks = q.chunks;
  a.parts = q.parts; a.PP = q.PP; a.work = q.work; a.row_count = q.row_count;
  a.part = (float*)ws;
}

template <typename T, int V, bool TAIL>
hipError_t norm_forward_v(const NormArgs<T>& a, const NormPlan& q, hipStream_t s) {
  const dim3 grid(q.blocks), block((unsigned)q.threads);
  if (q.row) { norm_row_kernel<T, V, TAIL><<<grid, block, 0, s>>>(a); return hipGetLastError(); }
#define ABS_NORM_F(NP_)                                                               \
  if (q.NP == NP_) {                                                                  \
    if (q.split) norm_forward_kernel<T, V, NP_, false, TAIL><<<grid, block, 0, s>>>(a); \
    else         norm_forward_kernel<T, V, NP_, true, TAIL><<<grid, block, 0, s>>>(a);  \
  }
  ABS_NORM_F(1) ABS_NORM_F(4) ABS_NORM_F(16)
#undef ABS_NORM_F
  if (q.split) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    norm_apply_kernel<T, V, TAIL><<<grid, block, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, int V, bool TAIL>
hipError_t norm_backward_v(const NormArgs<T>& a, const NormPlan& q, hipStream_t s) {
  const dim3 grid(q.blocks), block((unsigned)q.threads);
  if constexpr (V == 4 && !TAIL) {
    if (q.row) { norm_row_backward_kernel<T, V><<<grid, block, 0, s>>>(a); return hipGetLastError(); }
  }
  const int stack = q.threads / std::max(q.TX, 64);
  const size_t lds = q.NP * V >= 32          ? (size_t)q.threads * V * 8        // (kLean; 32 KB at most either way)
                     : a.rows_g && stack > 1 ? (size_t)stack * V * q.TX * 4 : 0;
  if constexpr (V == 8) {                                      // (single positions, never split)
    norm_backward_kernel<T, V, 1, true, TAIL><<<grid, block, lds, s>>>(a);
    return hipGetLastError();
  } else {
#define ABS_NORM_B(NP_)                                                                    \
  if (q.NP == NP_) {                                                                       \
    if (q.split) norm_backward_kernel<T, V, NP_, false, TAIL><<<grid, block, lds, s>>>(a);  \
    else         norm_backward_kernel<T, V, NP_, true, TAIL><<<grid, block, lds, s>>>(a);   \
  }
    ABS_NORM_B(1) ABS_NORM_B(4) ABS_NORM_B(8)
#undef ABS_NORM_B
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && q.split) {
      const dim3 all(std::min(a.work, 1u << 20));
      norm_backward_apply_kernel<T, V, TAIL><<<all, block, 0, s>>>(a);
      e = hipGetLastError();
    }
    return e;
  }
}

template <typename T, int V, bool TAIL>
hipError_t norm_either(bool backward, const NormArgs<T>& a, const NormPlan& q, hipStream_t s) {
  return backward ? norm_backward_v<T, V, TAIL>(a, q, s) : norm_forward_v<T, V, TAIL>(a, q, s);
}

template <typename T>
hipError_t norm_run(const abs_group_norm& p, bool backward, NormArgs<T> a, const NormPlan& q, char* ws, float* dgamma, float* dbeta,
                    hipStream_t s) {
  norm_fill(a, p, q, ws);
  if (backward && dgamma) {
    const bool one = q.row_count == 1;
    a.rows_g = one ? dgamma : (float*)(ws + q.off_rows);
    a.rows_b = one ? dbeta : a.rows_g + p.channels;
    a.row_step = 2 * (int64_t)p.channels;
  }
  hipError_t e = hipSuccess;
  if (q.plain) {
    if (backward) {
      if (a.rows_g) {
        norm_plain_share_kernel<T><<<dim3((unsigned)((p.channels + 255) / 256), q.row_count), 256, 0, s>>>(a);
        e = hipGetLastError();
      }
      if (e == hipSuccess) { norm_plain_kernel<T, true><<<dim3(q.blocks), 1024, 0, s>>>(a); e = hipGetLastError(); }
    } else {
      norm_plain_kernel<T, false><<<dim3(q.blocks), 1024, 0, s>>>(a);
      e = hipGetLastError();
    }
  } else {
    switch (q.V) {
      case 8:
        if constexpr (sizeof(T) == 2) e = norm_either<T, 8, false>(backward, a, q, s);
        break;
      case 4: e = q.tail ? norm_either<T, 4, true>(backward, a, q, s) : norm_either<T, 4, false>(backward, a, q, s); break;
      case 2: e = q.tail ? norm_either<T, 2, true>(backward, a, q, s) : norm_either<T, 2, false>(backward, a, q, s); break;
      default: e = norm_either<T, 1, false>(backward, a, q, s);
    }
  }
  if (e == hipSuccess && a.rows_g && q.row_count > 1) {
    norm_share_sum_kernel<<<dim3((unsigned)((p.channels + 31) / 32), 2), 1024, 0, s>>>(a.rows_g, q.row_count, p.channels, dgamma, dbeta);
    e = hipGetLastError();
  }
  return e;
}

__global__ void norm_zero_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) { a[i] = 0.f; b[i] = 0.f; }
}

}  // namespace
}  // namespace abs_impl

using namespace abs_impl;

extern "C" {

size_t abs_group_norm_workspace_size(const abs_group_norm* p, int32_t backward) {
  if (const char* why = norm_problem(p, backward != 0)) { op_fail(ABS_E_ARG, why); return 0; }
  return p->n ? norm_plan(*p, backward != 0, norm_piece(*p, backward != 0)).bytes : 0;
}

int abs_group_norm_forward(const abs_group_norm* p, const void* d_x, const float* d_gamma, const float* d_beta,
                           void* d_y, float* d_mean, float* d_rstd, void* d_workspace, size_t workspace_bytes,
                           void* hip_stream) {
  if (const char* why = norm_problem(p, false)) return op_fail(ABS_E_ARG, why);
  if (!d_gamma != !d_beta) return op_fail(ABS_E_ARG, "group norm: gamma and beta come together");
  if (!d_mean != !d_rstd) return op_fail(ABS_E_ARG, "group norm: mean and rstd come together");
  if (p->n == 0) return ABS_OK;
  if (!d_x || !d_y) return op_fail(ABS_E_ARG, "group norm: a device pointer is NULL");
  const uintptr_t all = (uintptr_t)d_x | (uintptr_t)d_y;
  if (all & (uintptr_t)(op_size(p->dtype) - 1) || ((uintptr_t)d_gamma | (uintptr_t)d_beta | (uintptr_t)d_mean | (uintptr_t)d_rstd) & 3)
    return op_fail(ABS_E_ARG, "group norm: a pointer is not aligned to its elements");
  const NormPlan q = norm_plan(*p, false, norm_piece(*p, false));
  if (q.bytes && (!d_workspace || (uintptr_t)d_workspace & 255)) return op_fail(ABS_E_ARG, "group norm: d_workspace must be 256-byte aligned");
  if (workspace_bytes < q.bytes) return op_fail(ABS_E_WORKSPACE, "group norm: workspace too small");
  hipError_t e;
  if (p->dtype == ABS_X_BF16) {
    NormArgs<uint16_t> a{};
    a.x = (const uint16_t*)d_x; a.y = (uint16_t*)d_y; a.ldy = p->ldy;
    a.gamma = d_gamma; a.beta = d_beta; a.mean = d_mean; a.rstd = d_rstd;
    e = norm_run(*p, false, a, q, (char*)d_workspace, nullptr, nullptr, (hipStream_t)hip_stream);
  } else {
    NormArgs<float> a{};
    a.x = (const float*)d_x; a.y = (float*)d_y; a.ldy = p->ldy;
    a.gamma = d_gamma; a.beta = d_beta; a.mean = d_mean; a.rstd = d_rstd;
    e = norm_run(*p, false, a, q, (char*)d_workspace, nullptr, nullptr, (hipStream_t)hip_stream);
  }
  return op_hip("abs_group_norm_forward", e);
}

int abs_group_norm_backward(const abs_group_norm* p, const void* d_x, const float* d_gamma, const float* d_beta,
                            const float* d_mean, const float* d_rstd, const void* d_dy, const void* d_dres,
                            void* d_dx, float* d_dgamma, float* d_dbeta, void* d_workspace, size_t workspace_bytes,
                            void* hip_stream) {
  if (const char* why = norm_problem(p, true)) return op_fail(ABS_E_ARG, why);
  if (!d_gamma != !d_beta) return op_fail(ABS_E_ARG, "group norm: gamma and beta come together");
  if (!d_dgamma != !d_dbeta) return op_fail(ABS_E_ARG, "group norm: dgamma and dbeta come together");
  if (d_dres && (p->lddres < p->channels || p->lddres >= 1ll << 40)) return op_fail(ABS_E_ARG, "group norm: a pitch is below channels");
  const uintptr_t f = (uintptr_t)d_gamma | (uintptr_t)d_beta | (uintptr_t)d_mean | (uintptr_t)d_rstd | (uintptr_t)d_dgamma | (uintptr_t)d_dbeta;
  const uintptr_t all = (uintptr_t)d_x | (uintptr_t)d_dy | (uintptr_t)d_dx | (uintptr_t)d_dres;
  if (all & (uintptr_t)(op_size(p->dtype) - 1) || f & 3) return op_fail(ABS_E_ARG, "group norm: a pointer is not aligned to its elements");
  if (p->n == 0) {
    if (!d_dgamma) return ABS_OK;
    norm_zero_kernel<<<dim3((unsigned)((p->channels + 255) / 256)), 256, 0, (hipStream_t)hip_stream>>>(d_dgamma, d_dbeta, p->channels);
    return op_hip("abs_group_norm_backward", hipGetLastError());
  }
  if (!d_x || !d_dy || !d_dx || !d_mean || !d_rstd) return op_fail(ABS_E_ARG, "group norm: a device pointer is NULL");
  const NormPlan q = norm_plan(*p, true, norm_piece(*p, true));
  if (q.bytes && (!d_workspace || (uintptr_t)d_workspace & 255)) return op_fail(ABS_E_ARG, "group norm: d_workspace must be 256-byte aligned");
  if (workspace_bytes < q.bytes) return op_fail(ABS_E_WORKSPACE, "group norm: workspace too small");
  hipError_t e;
  if (p->dtype == ABS_X_BF16) {
    NormArgs<uint16_t> a{};
    a.x = (const uint16_t*)d_x; a.dy = (const uint16_t*)d_dy; a.dres = (const uint16_t*)d_dres; a.y = (uint16_t*)d_dx;
    a.ldy = p->lddx; a.lddy = p->lddy; a.lddres = p->lddres;
    a.gamma = d_gamma; a.beta = d_beta; a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
    e = norm_run(*p, true, a, q, (char*)d_workspace, d_dgamma, d_dbeta, (hipStream_t)hip_stream);
  } else {
    NormArgs<float> a{};
    a.x = (const float*)d_x; a.dy = (const float*)d_dy; a.dres = (const float*)d_dres; a.y = (float*)d_dx;
    a.ldy = p->lddx; a.lddy = p->lddy; a.lddres = p->lddres;
    a.gamma = d_gamma; a.beta = d_beta; a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
    e = norm_run(*p, true, a, q, (char*)d_workspace, d_dgamma, d_dbeta, (hipStream_t)hip_stream);
  }
  return op_hip("abs_group_norm_backward", e);
}

}  // extern "C"
