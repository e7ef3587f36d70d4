// RMS norms of the query and key heads and their rotation by position, in one
// pass over the q and k columns of the fused projection; forward and backward.
//
// A row x of dh elements is one head of one token. With r = 1 / sqrt(mean(x^2) + eps)
// and the gain g of its kind (query or key), n = x r g; the first R elements of n
// form R / 2 pairs (a, b), and pair i turns by the angle t_i = pos * freq[i]:
//   y = (a cos t - b sin t, a sin t + b cos t); the other elements pass through.
// The rotation is orthogonal, so the backward turns dy back by the same angle,
// dn = rot(dy, -t), and with xh = x r, e = dn g:
//   dg = sum over tokens and heads of dn xh,   dx = r (e - xh mean(e xh)).
//
// Bound by HBM: 2 (forward) or 3 (backward) elements moved per element, some
// 10 flop each. So a lane owns 16 elements of a row as two 8-element vectors that
// hold both members of 8 pairs (half layout: elements 8 i and R / 2 + 8 i; adjacent
// layout: 16 consecutive ones), dh / 16 lanes own a row, the sums of a row are
// row-local lane moves, and a pair never crosses lanes. The lanes of a token (all
// its heads) are the `slots`; a thread keeps its slot over all its tokens, so its
// gains and, in the backward, its sums for the gains and for the column sums of
// dx stay in registers. The tokens of a workgroup are taken U to a thread at a
// time: their loads are issued first, then the workgroup computes the angles of
// those tokens once for all heads, into LDS. Measured, a pass over 8192 tokens of 16 + 16
// heads of 64 in bf16: forward 15.2 us on one set of buffers, part of which stays in the
// 256 MB cache (a copy of the same 67 MB: 10.2), 19.0 on eight sets in turn, from HBM
// (copy 14.1); backward 28.6 and 34.2 us, 4 of them the sums' second launch.
//
// Angles: pos * freq in 64 bits and reduced to a fraction of a turn there (a 32-bit
// product is off by 0.06 at position 10^6); the sine and cosine of the fraction
// in 32 bits.
//
// The backward's sums leave a workgroup as one row of partial sums in the
// workspace; a second launch adds the rows in order, so results do not depend on
// the order in which workgroups run.
#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"

namespace paci {
namespace {

constexpr int NT = 256;       // threads of a workgroup that takes whole tokens
constexpr int NT_MAX = 512;   // of one that takes a part of a token's heads, or wide tokens in the backward

struct RotKernelArgs {
  const void* x; int64_t ldx;
  const void* dy; int64_t lddy;
  void* out; int64_t ldout;
  const float* gain_q;
  const float* gain_k;
  const int32_t* pos;
  const double* freq;
  float* part_bias;   // [gridDim.x][(Hq + Hk) dh], or null
  float* part_gain;   // [gridDim.x * gridDim.y][2 dh]
  int T, seq, Hq, Hk, dh, R;
  int slots, part, par;   // lanes of a token, those of them that one workgroup takes, its tokens side by side
  int chunks;         // ceil(T / (U * par))
  float eps, inv_dh;
  int adjacent;
};

// Sum over the LPR lanes of a row (LPR lanes in line, a power of two up to 16).
template <int LPR> __device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (LPR >= 2) v += dpp_f<0xB1>(v);
  if constexpr (LPR >= 4) v += dpp_f<0x4E>(v);
  if constexpr (LPR >= 8) v += dpp_f<0x141>(v);
  if constexpr (LPR >= 16) v += dpp_f<0x140>(v);
  return v;
}

// 8 consecutive elements as 16-byte vectors.
template <typename T> struct Oct { u32x4 v[8 * sizeof(T) / 16]; };
template <typename T> __device__ __forceinline__ Oct<T> ld_oct(const T* p) {
  Oct<T> o;
#pragma unroll
  for (int i = 0; i < 8 * (int)sizeof(T) / 16; ++i) o.v[i] = ld16g(p + i * (16 / sizeof(T)));
  return o;
}
template <typename T> __device__ __forceinline__ float oget(const Oct<T>& o, int j) {
  constexpr int V = Vec<T>::V;
  return vget<T>(o.v[j / V], j % V);
}
template <typename T> __device__ __forceinline__ void st_oct(T* p, const float* f);
template <> __device__ __forceinline__ void st_oct<float>(float* p, const float* f) {
  st16g(p, __builtin_bit_cast(u32x4, floatx4{f[0], f[1], f[2], f[3]}));
  st16g(p + 4, __builtin_bit_cast(u32x4, floatx4{f[4], f[5], f[6], f[7]}));
}
template <> __device__ __forceinline__ void st_oct<bf16>(bf16* p, const float* f) {
  st16g(p, u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])});
}

// Turns the 8 pairs of a lane by the angles cs (cos, sin); SIGN -1 turns back.
// f[0..7] is the lane's first vector, f[8..15] its second.
template <int SIGN> __device__ __forceinline__ void rotate(float (&f)[16], const float2* cs, bool adjacent) {
  floatx4 c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = reinterpret_cast<const floatx4*>(cs)[i];
  if (adjacent) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float co = c[i >> 1][2 * (i & 1)], si = SIGN * c[i >> 1][2 * (i & 1) + 1];
      const float a = f[2 * i], b = f[2 * i + 1];
      f[2 * i] = a * co - b * si;
      f[2 * i + 1] = a * si + b * co;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float co = c[i >> 1][2 * (i & 1)], si = SIGN * c[i >> 1][2 * (i & 1) + 1];
      const float a = f[i], b = f[8 + i];
      f[i] = a * co - b * si;
      f[8 + i] = a * si + b * co;
    }
  }
}

// LPR: lanes reserved for a row, dh / 16 rounded up to a power of two.
// U: tokens of a thread in flight.
template <typename T, int LPR, int U, bool NORM, bool BWD>
__global__ void __launch_bounds__(NT_MAX) rotary_kernel(RotKernelArgs a) {
  extern __shared__ floatx4 lds[];   // angles [U * par][R / 2] (cos, sin), two buffers in the backward; then its sums, 32 floats a thread
  const int tid = threadIdx.x, nt = blockDim.x;
  const int R2 = a.R / 2;
  const int p = tid / a.part;                                   // the thread's token within the workgroup
  const int slot = blockIdx.y * a.part + (tid - p * a.part);
  const int row = slot / LPR, i = slot % LPR;
  const bool live = p < a.par && slot < a.slots && 16 * i < a.dh;
  const bool turned = 16 * i < a.R;
  int oa, ob;   // element offsets of the lane's two vectors in the row
  if (a.adjacent) {
    oa = 16 * i;
    ob = oa + 8;
  } else if (turned) {
    oa = 8 * i;
    ob = R2 + 8 * i;
  } else {
    oa = a.R + 8 * (i - a.R / 16);
    ob = oa + (a.dh - a.R) / 2;
  }
  const int64_t ca = (int64_t)row * a.dh + oa, cb = (int64_t)row * a.dh + ob;
  const T* x = reinterpret_cast<const T*>(a.x);
  const T* dy = reinterpret_cast<const T*>(a.dy);
  T* out = reinterpret_cast<T*>(a.out);

  float g[16], sg[16], sb[16];
  if constexpr (NORM) {
    const float* gain = row < a.Hq ? a.gain_q : a.gain_k;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[j] = live ? gain[oa + j] : 0.f;
      g[8 + j] = live ? gain[ob + j] : 0.f;
    }
  }
  if constexpr (BWD) {
#pragma unroll
    for (int j = 0; j < 16; ++j) sg[j] = sb[j] = 0.f;
  }
  const int TB = U * a.par;   // tokens of a chunk
  int buf = 0;
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x, buf ^= 1) {
    const int t0 = c * TB;
    Oct<T> xa[U], xb[U], ya[U], yb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * a.par + p;
      if (live && t < a.T) {
        if constexpr (NORM || !BWD) {
          const T* xr = x + (int64_t)t * a.ldx;
          xa[u] = ld_oct(xr + ca);
          xb[u] = ld_oct(xr + cb);
        }
        if constexpr (BWD) {
          const T* yr = dy + (int64_t)t * a.lddy;
          ya[u] = ld_oct(yr + ca);
          yb[u] = ld_oct(yr + cb);
        }
      }
    }
    float2* cs = reinterpret_cast<float2*>(lds) + buf * TB * R2;
    if (R2 > 0) {
      for (int k = tid; k < TB * R2; k += nt) {
        const int tt = k / R2, fi = k - tt * R2;
        const int t = min(t0 + tt, a.T - 1);
        const int ps = a.pos != nullptr ? a.pos[t] : t % a.seq;
        const double turns = (double)ps * (a.freq[fi] * 0.15915494309189533577);
        const float f = (float)(turns - __builtin_rint(turns));
        float si, co;
        sincospif(2.f * f, &si, &co);
        cs[k] = make_float2(co, si);
      }
      __syncthreads();   // the other buffer is read until the next chunk's barrier
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * a.par + p;
      const bool ok = live && t < a.T;
      const float2* ang = cs + (u * a.par + (p < a.par ? p : 0)) * R2 + 8 * i;
      float f[16];
      if constexpr (!BWD) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[j] = ok ? oget(xa[u], j) : 0.f;
          f[8 + j] = ok ? oget(xb[u], j) : 0.f;
        }
        if constexpr (NORM) {
#pragma unroll
          for (int j = 0; j < 16; ++j) ss += f[j] * f[j];
          const float r = rsqrtf(lanes_sum<LPR>(ss) * a.inv_dh + a.eps);
#pragma unroll
          for (int j = 0; j < 16; ++j) f[j] = f[j] * r * g[j];
        }
        if (ok && turned) rotate<1>(f, ang, a.adjacent);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[j] = ok ? oget(ya[u], j) : 0.f;
          f[8 + j] = ok ? oget(yb[u], j) : 0.f;
        }
        if (ok && turned) rotate<-1>(f, ang, a.adjacent);
        if constexpr (NORM) {
          float xh[16], ss = 0.f, dot = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            xh[j] = ok ? oget(xa[u], j) : 0.f;
            xh[8 + j] = ok ? oget(xb[u], j) : 0.f;
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) ss += xh[j] * xh[j];
          const float r = rsqrtf(lanes_sum<LPR>(ss) * a.inv_dh + a.eps);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            xh[j] *= r;
            sg[j] += f[j] * xh[j];
            f[j] *= g[j];
            dot += f[j] * xh[j];
          }
          const float m = lanes_sum<LPR>(dot) * a.inv_dh;
#pragma unroll
          for (int j = 0; j < 16; ++j) f[j] = r * (f[j] - xh[j] * m);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) sb[j] += f[j];
      }
      if (ok) {
        T* o = out + (int64_t)t * a.ldout;
        st_oct(o + ca, f);
        st_oct(o + cb, f + 8);
      }
    }
  }
  if constexpr (BWD) {
    // Sums of the workgroup, in halving rounds: the upper half of the members leaves its sums in
    // LDS, the lower half adds them (a round's writers are none of the round before's readers'
    // sources, so one barrier a round). First the tokens side by side; then the column sums are
    // whole, and the gains' add up over the heads of their kind.
    floatx4* red = lds;   // [thread][4] of sb, then of sg; units rotated by the thread against bank conflicts
    auto put = [&](const float (&v)[16], int part) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        red[(part * nt + tid) * 4 + ((q + (tid >> 1)) & 3)] = floatx4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    };
    auto add = [&](float (&v)[16], int part, int from) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4 u = red[(part * nt + from) * 4 + ((q + (from >> 1)) & 3)];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[4 * q + r] += u[r];
      }
    };
    auto out16 = [&](float* to, const float (&v)[16]) {   // the thread's columns of a row
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<floatx4*>(to + (q < 2 ? oa : ob) + 4 * (q & 1)) =
            floatx4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    };
    const bool bias = a.part_bias != nullptr;
    if (NORM || bias) {
      __syncthreads();   // the angles' last readers
      for (int n = a.par, half; n > 1; n = half) {
        half = (n + 1) / 2;
        if (p >= half && p < n) {
          if (bias) put(sb, 0);
          if (NORM) put(sg, 1);
        }
        __syncthreads();
        if (p < n - half) {
          if (bias) add(sb, 0, tid + half * a.part);
          if (NORM) add(sg, 1, tid + half * a.part);
        }
      }
    }
    if (bias && live && p == 0) out16(a.part_bias + ((int64_t)blockIdx.x * (a.Hq + a.Hk) + row) * a.dh, sb);
    if constexpr (NORM) {
      const int row0 = blockIdx.y * a.part / LPR;                        // first row of this workgroup
      const int rows = min(a.part, a.slots - (int)blockIdx.y * a.part) / LPR;
      const int nq = min(max(a.Hq - row0, 0), rows), nk = rows - nq;
      const bool key = row >= a.Hq;
      const int idx = row - row0 - (key ? nq : 0), len = key ? nk : nq;   // among the rows of its kind
      for (int n = max(nq, nk), half; n > 1; n = half) {
        half = (n + 1) / 2;
        const int end = p == 0 ? min(n, len) : 0;
        if (idx >= half && idx < end) put(sg, 1);
        __syncthreads();
        if (idx + half < end) add(sg, 1, tid + half * LPR);
      }
      if (live && p == 0 && idx == 0) {
        float* to = a.part_gain + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.dh;
        out16(to + (key ? a.dh : 0), sg);
        if (len == rows) {   // no head of the other kind here
#pragma unroll
          for (int j = 0; j < 16; ++j) sg[j] = 0.f;
          out16(to + (key ? 0 : a.dh), sg);
        }
      }
    }
  }
}

// out[c] += sum over the rows of part [rows][cols], rows in a fixed order: 16
// columns and 16 row groups to a workgroup. The columns are those of the bias
// (cols_b, over rows_b), then of the two gains (2 dh, over rows_g).
__global__ void __launch_bounds__(NT) rotary_sums_kernel(const float* __restrict__ part_b, int rows_b, int cols_b,
                                                          float* out_b, const float* __restrict__ part_g, int rows_g,
                                                          int dh, float* out_q, float* out_k) {
  __shared__ float red[16][17];
  const int nb = (cols_b + 15) / 16;
  const bool gain = (int)blockIdx.x >= nb;
  const float* part = gain ? part_g : part_b;
  const int cols = gain ? 2 * dh : cols_b, rows = gain ? rows_g : rows_b;
  const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int col = ((int)blockIdx.x - (gain ? nb : 0)) * 16 + cl;
  float s = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int r = rg; r < rows; r += 16) s += part[(int64_t)r * cols + col];
  }
  red[rg][cl] = s;
  __syncthreads();
  if (rg != 0 || col >= cols) return;
  for (int r = 1; r < 16; ++r) s += red[r][cl];
  float* out = !gain ? out_b : col < dh ? out_q : out_k;
  if (out != nullptr) out[gain && col >= dh ? col - dh : col] += s;
}

// The launch of a pass. U tokens in flight per thread: 128 bytes a lane in the forward
// (4 tokens in bf16, 2 in fp32), half that in the backward, which reads two rows and
// holds its sums (with 4 it takes 256 registers and spills to the second file: 13 us more
// at 8192 tokens of 16 + 16 heads of 64 in bf16; 1 is as fast there). Backward workgroups
// each leave a row of sums, so there are few: two of 256 threads to a CU (27.4 us there;
// one 30.6, three 32.4), or one of up to 512 where a token has 128 lanes or more. us with
// two of 256 / one of 512: 8192 tokens of 16 + 16 heads of 64: 27.4 / 26.7, in fp32 39.6 /
// 39.6; of 128: 43.7 / 42.8, 86.4 / 84.4; 32768 of 32 + 8 heads of 128: 227 / 219; 4096 of
// 32 + 8 in fp32: 56.1 / 50.7; but 12 + 12 heads of 64: 24.4 / 25.5, 16384 tokens of 8 + 2
// heads of 96: 30.8 / 31.2.
struct RotPlan {
  int lpr, slots, part, par, U, chunks, threads, gx, gy;
  size_t lds;
};
constexpr size_t kAngleBytes = 65536;   // LDS for angles: two workgroups to a CU at least
RotPlan rot_plan(const RotArgs& r, bool bwd) {
  RotPlan p;
  for (p.lpr = 1; 16 * p.lpr < r.dh;) p.lpr *= 2;
  const int rows = r.q_heads + r.k_heads;
  p.slots = rows * p.lpr;
  const bool wide = bwd && p.slots >= NT / 2;
  const int nt = wide ? NT_MAX : NT, per_cu = wide ? 1 : 2;
  // a token's heads in as few workgroups as hold them, evenly; several tokens side by side if they are few
  p.gy = p.slots <= nt ? 1 : (p.slots + NT_MAX - 1) / NT_MAX;
  p.part = (rows + p.gy - 1) / p.gy * p.lpr;
  p.gy = (p.slots + p.part - 1) / p.part;
  p.par = std::max(1, nt / p.part);
  p.U = (r.dt == DT_BF16 ? 4 : 2) / (bwd ? 2 : 1);
  // the backward walks chunks with two buffers of angles, the forward takes one chunk per workgroup
  const size_t token = (size_t)(bwd ? 2 : 1) * (r.rope_dims / 2) * sizeof(float2);   // LDS per token
  if (token > 0) p.par = std::min<int64_t>(p.par, kAngleBytes / (token * p.U));
  p.par = std::min(p.par, r.T);
  // few tokens: one to a thread, so that the workgroups spread over the CUs
  if ((int64_t)((r.T + p.U * p.par - 1) / (p.U * p.par)) * p.gy < cu_count()) p.U = 1;
  p.chunks = (r.T + p.U * p.par - 1) / (p.U * p.par);
  p.gx = p.chunks;
  if (bwd) p.gx = std::min(p.chunks, std::max(1, per_cu * cu_count() / p.gy));
  p.threads = (p.par * p.part + 63) / 64 * 64;
  p.lds = token * p.U * p.par;
  if (bwd) p.lds = std::max(p.lds, (size_t)p.threads * 32 * sizeof(float));   // the sums at its end
  return p;
}

template <typename T, int LPR, int U, bool BWD>
hipError_t rot_launch(const RotKernelArgs& k, const RotPlan& p, bool norm, hipStream_t st) {
  auto f = norm ? rotary_kernel<T, LPR, U, true, BWD> : rotary_kernel<T, LPR, U, false, BWD>;
  hipLaunchKernelGGL(f, dim3(p.gx, p.gy), dim3(p.threads), p.lds, st, k);
  return hipGetLastError();
}
template <typename T, int LPR>
hipError_t rot_u(const RotKernelArgs& k, const RotPlan& p, bool norm, bool bwd, hipStream_t st) {
  constexpr int UF = sizeof(T) == 2 ? 4 : 2, UB = UF / 2;
  if (bwd) return p.U == 1 ? rot_launch<T, LPR, 1, true>(k, p, norm, st) : rot_launch<T, LPR, UB, true>(k, p, norm, st);
  return p.U == 1 ? rot_launch<T, LPR, 1, false>(k, p, norm, st) : rot_launch<T, LPR, UF, false>(k, p, norm, st);
}
template <typename T>
hipError_t rot_lpr(const RotKernelArgs& k, const RotPlan& p, bool norm, bool bwd, hipStream_t st) {
  switch (p.lpr) {
    case 1: return rot_u<T, 1>(k, p, norm, bwd, st);
    case 2: return rot_u<T, 2>(k, p, norm, bwd, st);
    case 4: return rot_u<T, 4>(k, p, norm, bwd, st);
    case 8: return rot_u<T, 8>(k, p, norm, bwd, st);
    case 16: return rot_u<T, 16>(k, p, norm, bwd, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

int64_t rotary_workspace_floats(const RotArgs& r) {
  if (r.T == 0) return 0;
  const RotPlan p = rot_plan(r, true);
  return (int64_t)p.gx * (r.q_heads + r.k_heads) * r.dh + (int64_t)p.gx * p.gy * 2 * r.dh;
}

hipError_t rotary(const RotArgs& r, bool bwd, hipStream_t st) {
  if (r.T == 0) return hipSuccess;
  const bool norm = r.norm;
  if (r.T < 0 || r.q_heads < 0 || r.k_heads < 0 || r.q_heads + r.k_heads < 1 || r.dh % 16 || r.dh < 16 || r.dh > 256 ||
      r.rope_dims % 16 || r.rope_dims < 0 || r.rope_dims > r.dh || r.seq < 1)
    return hipErrorInvalidValue;
  const RotPlan p = rot_plan(r, bwd);
  const int cols = (r.q_heads + r.k_heads) * r.dh;
  RotKernelArgs k;
  k.x = r.x;
  k.ldx = r.ldx;
  k.dy = r.dy;
  k.lddy = r.lddy;
  k.out = r.out;
  k.ldout = r.ldout;
  k.gain_q = r.gain_q;
  k.gain_k = r.gain_k;
  k.pos = r.pos;
  k.freq = r.freq;
  k.part_bias = bwd && r.g_bias ? r.ws : nullptr;
  k.part_gain = bwd ? r.ws + (int64_t)p.gx * cols : nullptr;
  k.T = r.T;
  k.seq = r.seq;
  k.Hq = r.q_heads;
  k.Hk = r.k_heads;
  k.dh = r.dh;
  k.R = r.rope_dims;
  k.slots = p.slots;
  k.part = p.part;
  k.par = p.par;
  k.chunks = p.chunks;
  k.eps = r.eps;
  k.inv_dh = 1.f / r.dh;
  k.adjacent = r.adjacent;
  hipError_t e = r.dt == DT_BF16 ? rot_lpr<bf16>(k, p, norm, bwd, st) : rot_lpr<float>(k, p, norm, bwd, st);
  if (e != hipSuccess || !bwd || (!norm && !r.g_bias)) return e;
  const int nb = r.g_bias ? (cols + 15) / 16 : 0, ng = norm ? (2 * r.dh + 15) / 16 : 0;
  hipLaunchKernelGGL(rotary_sums_kernel, dim3(nb + ng), dim3(NT), 0, st, k.part_bias, p.gx, r.g_bias ? cols : 0, r.g_bias,
                     k.part_gain, p.gx * p.gy, r.dh, r.g_gain_q, r.g_gain_k);
  return hipGetLastError();
}

}  // namespace paci
