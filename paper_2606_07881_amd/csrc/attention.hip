// Causal multi-head attention, forward and backward, gfx950.
//
// q, k and v are rows of H * dh elements with a row stride each (side by side in
// the fused projection, or q and k in a buffer of their own) and are read in
// place. Blocks of 64 keys (and of 64 queries) are staged in LDS, and every
// product is an MFMA chain in the convention of device_common.hpp.
//
// Forward (one workgroup per (sequence, head, 64 queries); 4 wavefronts of 16
// queries, heaviest causal blocks first): S^T = K Q^T, so each lane owns one
// query and its per-query statistics stay lane-local. Online softmax runs in
// base 2 with the 1/sqrt(dh) * log2(e) scale folded in. O^T += V^T P^T takes
// P straight from the S^T accumulators (AccPerm order); V^T is staged
// transposed in that same order. The saved statistic is
// lse2 = max + log2(sum), in log2 units of the scaled scores.
//
// Backward: D = rowsum(dO * O) first. Then two kinds of workgroup, in one launch,
// recompute P from q, k and lse2, so neither needs atomics:
//   dK/dV  (per 64 keys; 16 keys per wavefront):  S = Q K^T and dP = dO V^T
//          with the key in the lane, dV^T += dO^T P, dK^T += Q^T dS;
//   dQ     (per 64 queries; 16 per wavefront):   S^T and dP^T with the query
//          in the lane, dQ^T += K^T dS^T.
#include <type_traits>

#include "device_common.hpp"
#include "kernels.hpp"

namespace paci {
namespace {

constexpr int NT = 256;
constexpr int BKV = 64;   // keys per block
constexpr float LOG2E = 1.4426950408889634f;

// Operands: row t of q at q + t * ldq (elements), head h at + h * dh; likewise k and v.
template <typename T> struct QkvView {
  const T* q; const T* k; const T* v;
  int64_t ldq, ldk, ldv;
};
// Gradients in the same manner, and where their column sums are added (H * dh floats each, nullable).
template <typename T> struct GradView {
  T* q; T* k; T* v;
  int64_t ldq, ldk, ldv;
  float* sq; float* sk; float* sv;
};

// ---- relative position bias -------------------------------------------------------------
// The score of query i and key j <= i adds table[bucket(i - j)][h], where distances
// from max_distance on share the last bucket reached. A workgroup serves one head, so
// its bias is a vector over the distance, built once in LDS in the units of q . k:
//   vec[FRONT + n] = sqrt(dh) * table[bucket(n)][h],  n = 0 .. max_distance, then the
//   value of max_distance up to n = max_distance + TAIL.
// The products of a tile start from it instead of from zero (the matrix instruction's
// third operand), so adding it costs no vector instruction.
// A tile of 16 queries and 16 keys at distance 16 D holds distances 16 D - 15 .. 16 D + 15,
// so tiles of equal D read the same values. A block whose distances all reach max_distance
// reads the last value everywhere; a path of its own for such blocks, with the one value in
// the exponent's constant, was no faster (backward 116 against 113 us at 8 x 1024 tokens, 16
// heads of 64; 385 against 372 at 4 x 2048, 16 heads of 128, max_distance 256).
// Entries at or below HIDDEN hide their distances (-inf), larger ones than MOST count as it.
// Both bounds are where the backward still holds: it forms P = 2^(x - lse2) from one float
// lse2, whose rounding is half a step at |entry| log2 e, so P is off by the factor
// 2^(2^-24 |lse2|) at worst: 1.0014 within 2^15 (a bf16 half step is 0.0039), 1.04 at 1e6, 6 at
// 1e8. (The forward's own error of that kind is in the sum as in its terms and cancels.)
struct BiasArgs {
  const float* table;      // [n_buckets][H]
  const int32_t* bounds;   // first distance of every bucket, ascending
  int n_buckets, max_distance;
  int batch;
  float* part;             // dQ wavefronts: sums of dS by distance, [H][batch][wavefront][max_distance + 1], or null
};
constexpr int BIAS_FRONT = 80, BIAS_TAIL = 128;   // distances below 0 (masked keys) and above max_distance inside a window
constexpr float BIAS_HIDDEN = -32768.f, BIAS_MOST = 32768.f;
__host__ __device__ __forceinline__ int bias_len(int max_distance) { return BIAS_FRONT + max_distance + BIAS_TAIL; }
// A dQ wavefront of SUB query tiles moves its diagonal sums through 4 rows of DiagRow floats of LDS.
template <int SUB> struct DiagRow { static constexpr int N = 16 * (SUB + 5), FLOATS = 4 * N; };
// LDS behind the tiles, floats: the vector, bounds and table column, then (dQ) the rows of each wavefront.
__host__ __device__ __forceinline__ int bias_lds_floats(int max_distance, int n_buckets, int diag) {
  return bias_len(max_distance) + 2 * n_buckets + diag;
}

// A query whose every key the bias hides has lse2 = -inf; +inf in its place makes every
// probability 2^(x - lse2) of the backward zero.
template <bool BIAS> __device__ __forceinline__ float query_lse(float lse2) {
  return BIAS && lse2 == -INFINITY ? INFINITY : lse2;
}

// A thread's bucket (thread index; at most 256 buckets): loaded ahead of the wait that covers
// the first tiles.
struct BiasEntry {
  float t;
  int bound;
};
__device__ __forceinline__ BiasEntry bias_load(const BiasArgs& a, int h, int H) {
  const int i = min((int)threadIdx.x, a.n_buckets - 1);
  return {a.table[(int64_t)i * H + h], a.bounds[i]};
}
// Builds vec for the head of the entries (every thread of the workgroup; NTH >= 256 threads;
// ends in a barrier).
template <int NTH, int DH> __device__ __forceinline__ void bias_build(float* vec, const BiasArgs& a, const BiasEntry& e) {
  static_assert(NTH >= MAX_BUCKETS, "a thread per bucket");
  int* bnd = reinterpret_cast<int*>(vec + bias_len(a.max_distance));
  float* col = vec + bias_len(a.max_distance) + a.n_buckets;
  if ((int)threadIdx.x < a.n_buckets) {
    const float t = (e.t > BIAS_MOST && e.t < INFINITY ? BIAS_MOST : e.t) * sqrtf((float)DH);
    bnd[threadIdx.x] = e.bound;
    col[threadIdx.x] = e.t <= BIAS_HIDDEN ? -INFINITY : t;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bias_len(a.max_distance); i += NTH) {
    const int n = min(max(i - BIAS_FRONT, 0), a.max_distance);
    int lo = 0, hi = a.n_buckets;   // the last bucket whose bound is at or below n (bucket 0 if none)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (bnd[mid] <= n) lo = mid;
      else hi = mid;
    }
    vec[i] = col[lo];
  }
  __syncthreads();
}

// Sums over the diagonals of dS, for the table's gradient: a dQ wavefront of 16 SUB
// queries adds up dS by distance and leaves one row of sums per distance in `part`
// (distances below max_distance; the last entry holds the rest), which a second
// launch adds by bucket in a fixed order.
//
// acc[i][r] of lane (g = l / 16, c = l % 16) is the sum over a block's tiles with
// qs - kt = i - 3 (query tile minus key tile), at distance D0 + 16 (i - 3) + c - 4 g - r,
// where D0 = first query - first key of the block. Moving the r-th value by r lanes
// within the 16 lines the four up (what leaves a row of lanes belongs to the window
// before). The lane groups' rows, 4 g apart, meet in LDS: six to eight stores and
// eight loads a block, where adding all four groups into one vector by LDS atomics
// took 19 us of a 143 us backward (8 x 1024 tokens, 16 heads of 64, max_distance 128),
// and this about 3.
// A block holds distances D0 - 63 .. D0 + 16 SUB - 1, and the next block's D0 is 64 less, so
// the sums of D0 + 1 .. D0 + 64 are complete with this block: lane j stores distance D0 + 1 + j,
// this block's part added to what the block before left there (carry).
template <int SUB> struct DiagSums {
  static constexpr int NB = SUB + 3, N = DiagRow<SUB>::N;
  float* rows;       // this wavefront's rows in LDS
  float* out;        // its row of part, or null
  int max_distance;
  float carry = 0.f, far = 0.f;   // sums of the block before; of distances from max_distance on

  __device__ __forceinline__ void init(float* lds, float* to, int md) {
    rows = lds + (threadIdx.x >> 6) * DiagRow<SUB>::FLOATS;
    out = to;
    max_distance = md;
    // the last 16 entries of a row stay zero (no tile reaches those distances)
    rows[(lane_id() >> 4) * N + N - 16 + (lane_id() & 15)] = 0.f;
  }
  __device__ __forceinline__ void put(int dist, float v) {
    if (dist >= max_distance) far += v;
    else if (dist >= 0) out[dist] = v;
  }
  // The block at D0; returns nothing, keeps the sums of D0 - 63 .. D0.
  __device__ __forceinline__ void block(int D0, const float (&acc)[NB][4]) {
    const int l = lane_id(), g = l >> 4, c = l & 15;
    float* to = rows + g * N + c;
#pragma unroll
    for (int i = -1; i < NB; ++i) {
      float u = 0.f;
      if (i >= 0) {   // lane c takes lane c + r (row_shl)
        const int k = i < 0 ? 0 : i;
        u = acc[k][0] + dpp_shift<0x101>(acc[k][1]) + dpp_shift<0x102>(acc[k][2]) + dpp_shift<0x103>(acc[k][3]);
      }
      if (i + 1 < NB) {   // lane c takes lane c + r - 16 of the next window (row_shr 16 - r)
        const int k = i + 1 < NB ? i + 1 : 0;
        u += dpp_shift<0x11F>(acc[k][1]) + dpp_shift<0x11E>(acc[k][2]) + dpp_shift<0x11D>(acc[k][3]);
      }
      to[16 * (i + 1)] = u;   // entry x of row g is distance D0 + x - 64 - 4 g
    }
    wave_lds_order();
    float low = 0.f, high = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) low += rows[q * N + 1 + l + 4 * q];     // D0 - 63 + l
    if (l < 16 * SUB - 1) {
#pragma unroll
      for (int q = 0; q < 4; ++q) high += rows[q * N + 65 + l + 4 * q]; // D0 + 1 + l
    }
    wave_lds_order();
    put(D0 + 1 + l, carry + high);
    carry = low;
  }
  // After the last block (at D0).
  __device__ __forceinline__ void finish(int D0) {
    put(D0 - 63 + lane_id(), carry);
    far = wave_sum(far);
    if (lane_id() == 0) out[max_distance] = far;
  }
};

// ---------------------------------------------------------------------------------------
template <typename T, int DH, bool DROP, bool BIAS>
__global__ void __launch_bounds__(NT) attn_fwd_kernel(QkvView<T> in, T* out, float* lse2, int S, int H, int d,
                                                       float scale_log2, DropArgs drop, BiasArgs bias) {
  extern __shared__ float bvec[];
  constexpr int V = Vec<T>::V;
  constexpr int BQ = 64;
  constexpr int DKV = DH / V;           // 16-byte vectors per head row
  constexpr int QSTEPS = DH / (4 * V);  // MFMA steps over the head dimension
  constexpr int PSTEPS = BKV / (4 * V); // MFMA steps over a key block
  __shared__ u32x4 sK[DKV * BKV];
  __shared__ u32x4 sVt[(BKV / V) * DH];

  const int nqb = (S + BQ - 1) / BQ;
  const int qb = nqb - 1 - blockIdx.x;
  const int bh = blockIdx.y, b = bh / H, h = bh % H;
  const int w = threadIdx.x >> 6, l = lane_id();
  const T* Qp = in.q + (int64_t)b * S * in.ldq + h * DH;
  const T* Kp = in.k + (int64_t)b * S * in.ldk + h * DH;
  const T* Vp = in.v + (int64_t)b * S * in.ldv + h * DH;
  const int q0 = qb * BQ;
  const int qrow = q0 + 16 * w + (l & 15);

  u32x4 qf[QSTEPS];
#pragma unroll
  for (int s = 0; s < QSTEPS; ++s) {
    const int kv = s * 4 + (l >> 4);
    qf[s] = (qrow < S) ? ld16(Qp + (int64_t)qrow * in.ldq + kv * V) : u32x4{0, 0, 0, 0};
  }
  if constexpr (BIAS) bias_build<NT, DH>(bvec, bias, bias_load(bias, h, H));
  floatx4 acc[DH / 16];
#pragma unroll
  for (int t = 0; t < DH / 16; ++t) acc[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  const int last_kb = min((q0 + BQ - 1) / BKV, (S - 1) / BKV);
  for (int kb = 0; kb <= last_kb; ++kb) {
    const int k0 = kb * BKV;
    __syncthreads();
    stage_kmajor<T, BKV, DKV, NT>(sK, Kp + (int64_t)k0 * in.ldk, in.ldk, S - k0);
    stage_mnmajor<T, DH, BKV / V, NT>(sVt, Vp + (int64_t)k0 * in.ldv, in.ldv, S - k0, typename AccPerm<T>::type());
    __syncthreads();

    floatx4 st[BKV / 16];
#pragma unroll
    for (int kt = 0; kt < BKV / 16; ++kt) {
      st[kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < QSTEPS; ++s) mma_step<T>(st[kt], lds_frag<BKV>(sK, s, kt * 16), qf[s]);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < BKV / 16; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = k0 + kt * 16 + 4 * (l >> 4) + r;
        float x = st[kt][r] * scale_log2;
        if constexpr (BIAS) x = (st[kt][r] + bvec[BIAS_FRONT + min(max(qrow - key, 0), bias.max_distance)]) * scale_log2;
        if (key > qrow || key >= S) x = -INFINITY;
        st[kt][r] = x;
        mx = fmaxf(mx, x);
      }
    mx = group4_max(mx);
    const float m_new = fmaxf(m_run, mx);
    const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
    const float alpha = exp2f(m_run - m_use);
    float rs = 0.f;
#pragma unroll
    for (int kt = 0; kt < BKV / 16; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = exp2f(st[kt][r] - m_use);
        st[kt][r] = p;
        rs += p;
      }
    rs = group4_sum(rs);
    l_run = l_run * alpha + rs;
    m_run = m_new;
    if constexpr (DROP) {   // dropout: the product uses P * keep * scale, the normalizer all of P
#pragma unroll
      for (int kt = 0; kt < BKV / 16; ++kt) {
        const uint32_t bits = drop_row4(drop, bh, qrow, k0 + kt * 16 + 4 * (l >> 4));
#pragma unroll
        for (int r = 0; r < 4; ++r) st[kt][r] = ((bits >> r) & 1) ? st[kt][r] * drop.scale : 0.f;
      }
    }
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) acc[t] *= alpha;
#pragma unroll
    for (int s = 0; s < PSTEPS; ++s) {
      const u32x4 pf = acc_to_frag<T>(st, s);
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) mma_step<T>(acc[t], lds_frag<DH>(sVt, s, t * 16), pf);
    }
  }
  if (qrow < S) {
    const float inv = BIAS && l_run == 0.f ? 0.f : 1.f / l_run;   // a bias of -inf can leave a query no key
    T* op = out + ((int64_t)b * S + qrow) * d + h * DH;
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) {
      const int c = t * 16 + 4 * (l >> 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) op[c + r] = from_f32<T>(acc[t][r] * inv);
    }
    if ((l >> 4) == 0) lse2[(int64_t)bh * S + qrow] = m_run + log2f(l_run);
  }
}

// ---------------------------------------------------------------------------------------
// bf16 kernels on an LDS ring. A block is 64 consecutive rows (keys or
// queries) of one head, [64][dh] bf16, copied by direct-to-LDS loads into a
// ring of NS stages so that the next blocks load while one is used. Row r's
// 16-byte chunk c sits at chunk c ^ blk_swz(r). Fragment reads (ds_read_b128)
// take 16 rows at one chunk per 16 lanes; transpose reads (ds_read_b64_tr_b16)
// take 4 rows x 2 chunks per 16 lanes, two lane groups (8 rows) per cycle. At
// 8 and 16 chunks per row the swizzle sends row bits 0, 2, 1 to chunk bits 0,
// 1, 2 (and row bit 0 also to chunk bit 3 at 16): both kinds of read then hit
// every LDS bank once per cycle, which bank-conflict counters confirm.
template <int CPR> __device__ __forceinline__ int blk_swz(int r) {
  if constexpr (CPR == 4) return (r >> 2) & 3;
  const int f = (r & 1) | (((r >> 2) & 1) << 1) | (((r >> 1) & 1) << 2);
  if constexpr (CPR == 8) return f;
  else return f | ((r & 1) << 3);
}
template <int CPR> __device__ __forceinline__ int blk_slot(int r, int c) { return r * CPR + (c ^ blk_swz<CPR>(r)); }

// MFMA operand: rows = block rows row0 + (l % 16), contracted = head dims of step s.
template <int CPR> __device__ __forceinline__ u32x4 blk_frag(const u32x4* blk, int s, int row0) {
  const int l = lane_id();
  return blk[blk_slot<CPR>(row0 + (l & 15), s * 4 + (l >> 4))];
}
// MFMA operand: rows = head dims dh0 + (l % 16), contracted = the 32 block rows
// of step s in StepPairPerm order (the order acc_to_frag gives accumulators).
template <int CPR> __device__ __forceinline__ u32x4 blk_frag_tr(const u32x4* blk, int s, int dh0) {
  const int l = lane_id(), g = l >> 4, c = l & 15;
  const bf16* base = reinterpret_cast<const bf16*>(blk);
  const int e = dh0 + 4 * (c & 3);
  const int r_lo = s * 32 + 4 * g + (c >> 2), r_hi = r_lo + 16;
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) i16x4*)(base + blk_slot<CPR>(r_lo, e >> 3) * 8 + (e & 7)));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) i16x4*)(base + blk_slot<CPR>(r_hi, e >> 3) * 8 + (e & 7)));
  const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
  return u32x4{a[0], a[1], b[0], b[1]};
}
// Issue this thread's loads of one block (rows src[0..63], row stride ld) into
// LDS byte address lds. Rows at or past rows_valid (>= 1) re-read the last
// valid row; every consumer masks those rows out.
template <int CPR, int NT>
__device__ __forceinline__ void blk_fill(const bf16* src, int64_t ld, int rows_valid, uint32_t lds, int w, int l) {
  constexpr int L = 64 * CPR / NT;
  static_assert(L >= 1 && (64 * CPR) % NT == 0, "block slots must split evenly over the threads");
#pragma unroll
  for (int p = 0; p < L; ++p) {
    const int blk = p * (NT / 64) + w;
    const int slot = blk * 64 + l;
    const int r = slot / CPR;
    const int c = (slot % CPR) ^ blk_swz<CPR>(r);
    const int rr = min(r, rows_valid - 1);
    dma16(src + (int64_t)rr * ld + c * 8, lds + (uint32_t)(blk * 1024));
  }
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)((const __attribute__((address_space(3))) char*)p);
}

// Forward, bf16: a workgroup takes 64 * QS * 4 queries, each wavefront 16 * QS
// of them (QS sub-tiles of 16, the query in the lane as in the kernel above),
// so every K and V fragment read from LDS feeds QS MFMAs. Key blocks are 64.
// SMALL: 64 queries, 16 to each of 4 wavefronts, for grids that would leave CUs
// idle: a workgroup walks its key blocks one after the other, so with less work
// per block it ends sooner. One sequence of 1024 keys, 12 heads of 64: 48
// workgroups, 27.1 us; 192 small ones, 16.6 (backward 28.7 -> 24.6); 2 x 200
// keys, 3 heads: 10.8 -> 6.1 (13.0 -> 10.9).
template <int DH, bool SMALL = false> struct FwdRing {
  static constexpr int CPR = DH / 8, KS = DH / 32;
  static constexpr int QS = SMALL ? 1 : DH == 32 ? 4 : (DH == 64 ? 2 : 1), WAVES = SMALL || DH == 32 ? 4 : 8,
                       NTF = 64 * WAVES;
  static constexpr int WQ = 16 * QS, BQ = WAVES * WQ;
  // blocks kb (V) and kb + 1 (K) are read in the same iteration, kb + 2 loads
  static constexpr int NS = 4;
  static constexpr int BLK = 64 * CPR;          // 16-byte slots per block
  static constexpr int L = 2 * BLK / NTF;       // loads per thread per stage (K and V)
};

// The key loop is software-pipelined (at head dim 64 and 128): while a
// wavefront runs the online softmax of key block kb on its vector ALUs, the
// MFMAs of the scores of block kb + 1 are interleaved with it, so the matrix
// unit is not idle during the exponentials. A wavefront's queries start at a multiple of 16 * QS, which
// divides 64, so every key block before its last one ends before its first
// query and inside the sequence: only the last block is masked.
template <int DH, bool DROP, bool SMALL, bool BIAS>
__global__ void __launch_bounds__((FwdRing<DH, SMALL>::NTF), 2) attn_fwd_ring_kernel(QkvView<bf16> in, bf16* out, float* lse2, int S, int H,
                                                               int d, float scale_log2, DropArgs drop, BiasArgs bias) {
  extern __shared__ float bvec[];
  using C = FwdRing<DH, SMALL>;
  constexpr int QS = C::QS, KS = C::KS, NS = C::NS, CPR = C::CPR;
  __shared__ u32x4 ring[NS * 2 * C::BLK];
  const int nqb = (S + C::BQ - 1) / C::BQ;
  const int qb = nqb - 1 - blockIdx.y;
  const int bh = blockIdx.x, b = bh / H, h = bh % H;
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4;
  const int wu = __builtin_amdgcn_readfirstlane(w);
  const bf16* Qp = in.q + (int64_t)b * S * in.ldq + h * DH;
  const bf16* Kp = in.k + (int64_t)b * S * in.ldk + h * DH;
  const bf16* Vp = in.v + (int64_t)b * S * in.ldv + h * DH;
  const int q0 = qb * C::BQ, qw0 = q0 + w * C::WQ;
  const uint32_t ring_lds = lds_addr(ring);
  const int nkb = min((q0 + C::BQ - 1) / BKV, (S - 1) / BKV) + 1;
  const int my_last = (qw0 < S) ? min((qw0 + C::WQ - 1) / BKV, (S - 1) / BKV) : -1;

  u32x4 qf[QS][KS];
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const int row = qw0 + 16 * qs + (l & 15);
#pragma unroll
    for (int s = 0; s < KS; ++s)
      qf[qs][s] = (row < S) ? ld16(Qp + (int64_t)row * in.ldq + s * 32 + 8 * g) : u32x4{0, 0, 0, 0};
  }
  floatx4 acc[QS][DH / 16];
  // the softmax normalizer: without dropout an MFMA of the probability
  // fragments against ones (the same bf16 P as the numerator, no cross-lane
  // sums); with dropout a running sum of all of P in fp32; with a bias, where the
  // statistic is an output, each lane's own fp32 sum, joined at the end
  floatx4 lacc[QS];
  const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};   // bf16 1.0 pairs
  float m_run[QS], l_run[QS];
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    m_run[qs] = -INFINITY;
    l_run[qs] = 0.f;
    lacc[qs] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) acc[qs][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  auto fill = [&](int kb) {
    const uint32_t st = ring_lds + (uint32_t)((kb % NS) * 2 * C::BLK * 16);
    const int k0 = kb * BKV;
    blk_fill<CPR, C::NTF>(Kp + (int64_t)k0 * in.ldk, in.ldk, S - k0, st, wu, l);
    blk_fill<CPR, C::NTF>(Vp + (int64_t)k0 * in.ldv, in.ldv, S - k0, st + C::BLK * 16, wu, l);
  };
  // raw scores q k^T of key block kb, with their bias
  auto scores = [&](int kb, floatx4 (&sc)[QS][4]) {
    const u32x4* sK = ring + (kb % NS) * 2 * C::BLK;
    floatx4 b[QS + 3];   // bias of the tiles' distances qs - kt
    if constexpr (BIAS) {
      const float* bp = bvec + BIAS_FRONT + min(qw0 - kb * BKV, bias.max_distance + 63) + (l & 15) - 4 * g;
#pragma unroll
      for (int i = 0; i < QS + 3; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) b[i][r] = bp[16 * (i - 3) - r];
    }
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      u32x4 kf[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[s] = blk_frag<CPR>(sK, s, kt * 16);
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) {
        if constexpr (BIAS) sc[qs][kt] = b[qs - kt + 3];
        else sc[qs][kt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) mma_step<bf16>(sc[qs][kt], kf[s], qf[qs][s]);
      }
    }
  };
  // online softmax of block kb's scores: running max and sum, rescaled
  // accumulators, and the probabilities (dropped ones zeroed) as bf16 fragments
  auto softmax = [&](auto masked, int kb, floatx4 (&sc)[QS][4], u32x4 (&pf)[QS][2]) {
    const int k0 = kb * BKV;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      const int qrow = qw0 + 16 * qs + (l & 15);
      if constexpr (decltype(masked)::value) {
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = k0 + kt * 16 + 4 * g + r;
            if (key > qrow || key >= S) sc[qs][kt][r] = -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[qs][kt][r]);
      mx = group4_max(mx);
      const float m_new = fmaxf(m_run[qs], mx * scale_log2);
      const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
      const float alpha = fast_exp2(m_run[qs] - m_use);
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[qs][kt][r] = fast_exp2(fmaf(sc[qs][kt][r], scale_log2, -m_use));
      if constexpr (BIAS) {
        float rs = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) rs += sc[qs][kt][r];
        l_run[qs] = l_run[qs] * alpha + rs;
      } else if constexpr (DROP) {
        float rs = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) rs += sc[qs][kt][r];
        l_run[qs] = l_run[qs] * alpha + group4_sum(rs);
      } else {
        lacc[qs] *= alpha;
      }
      m_run[qs] = m_new;
      if constexpr (DROP) {   // dropout: the product uses P * keep * scale, the normalizer all of P
#pragma unroll
        for (int kt = 0; kt < 4; kt += 2) {
          uint32_t bits[2];
          drop_row4_pair(drop, bh, qrow, k0 + kt * 16 + 4 * g, k0 + kt * 16 + 16 + 4 * g, bits[0], bits[1]);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              sc[qs][kt + u][r] = ((bits[u] >> r) & 1) ? sc[qs][kt + u][r] * drop.scale : 0.f;
        }
      }
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) acc[qs][t] *= alpha;
      pf[qs][0] = acc_to_frag<bf16>(sc[qs], 0);
      pf[qs][1] = acc_to_frag<bf16>(sc[qs], 1);
    }
  };
  auto pv = [&](int kb, const u32x4 (&pf)[QS][2]) {
    const u32x4* sV = ring + (kb % NS) * 2 * C::BLK + C::BLK;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) {
        const u32x4 vf = blk_frag_tr<CPR>(sV, s, t * 16);
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) mma_step<bf16>(acc[qs][t], vf, pf[qs][s]);
      }
    if constexpr (!DROP && !BIAS) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) mma_step<bf16>(lacc[qs], ones, pf[qs][s]);
    }
  };
  // iteration kb: blocks up to min(nkb - 1, kb + NS - 2) have been issued;
  // wait for block kb + 1, whose keys this iteration reads, then refill the
  // stage of block kb - 1, which every wavefront has finished with
  // (at 4 query sub-tiles per wavefront the two score arrays would not fit in
  // registers: that variant reads and computes block kb only)
  constexpr bool PIPE = QS <= 2;
  auto step = [&](int kb, floatx4 (&cur)[QS][4], floatx4 (&nxt)[QS][4]) {
    const int newest = PIPE ? kb + 1 : kb;   // the newest block this iteration reads
    if (newest < nkb) wait_loads<C::L, NS - 2>(min(nkb - 1, kb + NS - 2) - newest);
    wait_lds_reads();
    barrier_no_fence();
    if (kb + NS - 1 < nkb) fill(kb + NS - 1);
    if (kb > my_last) return;
    u32x4 pf[QS][2];
    if constexpr (!PIPE) {
      scores(kb, cur);
      if (kb < my_last) softmax(std::false_type{}, kb, cur, pf);
      else softmax(std::true_type{}, kb, cur, pf);
    } else if (kb < my_last) {
      scores(kb + 1, nxt);
      softmax(std::false_type{}, kb, cur, pf);
      // interleave: the fragment reads first, then one MFMA per few ALU instructions
      // (with a bias its reads too: 122 against 126 us a pass at 4 x 2048 tokens, 16 heads of 128)
      __builtin_amdgcn_sched_group_barrier(0x100, 4 * KS + (BIAS ? 2 * (QS + 3) : 0), 0);
#pragma unroll
      for (int i = 0; i < 4 * KS * QS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
      }
    } else {
      softmax(std::true_type{}, kb, cur, pf);
    }
    pv(kb, pf);
  };

  BiasEntry entry{};
  if constexpr (BIAS) entry = bias_load(bias, h, H);
#pragma unroll
  for (int t = 0; t < NS - 1; ++t)
    if (t < nkb) fill(t);
  floatx4 sA[QS][4], sB[QS][4];
  // every load so far, the query fragments included, through a wait the
  // compiler sees: it then knows qf has landed and puts no vmcnt(0) in the
  // loop, which would also wait for the ring's prefetches
  wait_vmcnt_all();
  if constexpr (BIAS) bias_build<C::NTF, DH>(bvec, bias, entry);
  barrier_no_fence();
  if (PIPE && my_last >= 0) scores(0, sA);
  for (int kb = 0; kb < nkb; kb += 2) {
    step(kb, sA, sB);
    if (kb + 1 < nkb) step(kb + 1, sB, sA);
  }
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const int qrow = qw0 + 16 * qs + (l & 15);
    if (qrow < S) {
      if constexpr (BIAS) l_run[qs] = group4_sum(l_run[qs]);
      else if constexpr (!DROP) l_run[qs] = lacc[qs][0];   // every row of the product holds the row sum
      const float inv = BIAS && l_run[qs] == 0.f ? 0.f : 1.f / l_run[qs];   // a bias of -inf can leave a query no key
      bf16* op = out + ((int64_t)b * S + qrow) * d + h * DH;
#pragma unroll
      for (int t = 0; t < DH / 16; ++t)
        *reinterpret_cast<u32x2*>(op + t * 16 + 4 * g) =
            u32x2{pack_bf16x2(acc[qs][t][0] * inv, acc[qs][t][1] * inv),
                  pack_bf16x2(acc[qs][t][2] * inv, acc[qs][t][3] * inv)};
      if (g == 0) lse2[(int64_t)bh * S + qrow] = m_run[qs] + log2f(l_run[qs]);
    }
  }
}

// D[bh][q] = sum_c dO[q][h*dh + c] * O[q][h*dh + c]; one wavefront per (token, head) row group.
template <typename T, int DH>
__global__ void __launch_bounds__(NT) attn_dsum_kernel(const T* o, const T* dO, float* D, int S, int H, int d,
                                                        int64_t rows) {
  constexpr int V = Vec<T>::V;
  constexpr int LPR = DH / V;  // lanes per (token, head) row
  const int64_t gid = (int64_t)blockIdx.x * NT + threadIdx.x;
  const int64_t row = gid / LPR;  // row = token * H + h
  const int part = gid % LPR;
  float s = 0.f;
  if (row < rows) {
    const int64_t tok = row / H;
    const int h = row % H;
    const int64_t off = tok * d + h * DH + part * V;
    const u32x4 a = ld16(o + off), g = ld16(dO + off);
#pragma unroll
    for (int j = 0; j < V; ++j) s += vget<T>(a, j) * vget<T>(g, j);
  }
#pragma unroll
  for (int w = LPR / 2; w >= 1; w >>= 1) s += __shfl_xor(s, w, 64);
  if (row < rows && part == 0) {
    const int64_t tok = row / H;
    const int h = row % H;
    const int64_t b = tok / S, q = tok % S;
    D[(b * H + h) * S + q] = s;
  }
}

// ---------------------------------------------------------------------------------------
// The fp32 backward's two kinds of workgroup (tiles: BwdTiles<T, DH>::SLOTS slots of LDS).
template <typename T, int DH> struct BwdTiles {
  static constexpr int BQ = 64;                      // queries per staged block of dK/dV
  static constexpr int TILE = DH / Vec<T>::V * 64;   // 64 rows of a head
  static constexpr int DKDV = 4 * DH / Vec<T>::V * BQ + BQ / 2, DQ = 3 * TILE;
  static constexpr int SLOTS = DKDV > DQ ? DKDV : DQ;
};
template <typename T, int DH, bool DROP, bool BIAS>
__device__ __forceinline__ void dkdv_body(u32x4* tiles, float* bvec, int kb, const QkvView<T>& in, const T* dO,
                                          const float* lse2, const float* Dsum, const GradView<T>& grad, int S, int H, int d,
                                          float scale_log2, float scale, const DropArgs& drop, const BiasArgs& bias) {
  constexpr int V = Vec<T>::V;
  constexpr int BQ = BwdTiles<T, DH>::BQ;
  constexpr int DKV = DH / V;
  constexpr int QSTEPS = DH / (4 * V);
  constexpr int RSTEPS = BQ / (4 * V);       // MFMA steps over a query block
  u32x4* sQ = tiles;
  u32x4* sdO = sQ + DKV * BQ;
  u32x4* sQt = sdO + DKV * BQ;
  u32x4* sdOt = sQt + (BQ / V) * DH;
  float* sL = reinterpret_cast<float*>(sdOt + (BQ / V) * DH);
  float* sD = sL + BQ;

  const int bh = blockIdx.y, b = bh / H, h = bh % H;
  const int w = threadIdx.x >> 6, l = lane_id();
  const T* Qp = in.q + (int64_t)b * S * in.ldq + h * DH;
  const T* Kp = in.k + (int64_t)b * S * in.ldk + h * DH;
  const T* Vp = in.v + (int64_t)b * S * in.ldv + h * DH;
  const T* dOp = dO + (int64_t)b * S * d + h * DH;
  const float* Lp = lse2 + (int64_t)bh * S;
  const float* Dp = Dsum + (int64_t)bh * S;
  const int k0 = kb * BKV;
  const int key = k0 + 16 * w + (l & 15);

  u32x4 kf[QSTEPS], vf[QSTEPS];
#pragma unroll
  for (int s = 0; s < QSTEPS; ++s) {
    const int kv = s * 4 + (l >> 4);
    kf[s] = (key < S) ? ld16(Kp + (int64_t)key * in.ldk + kv * V) : u32x4{0, 0, 0, 0};
    vf[s] = (key < S) ? ld16(Vp + (int64_t)key * in.ldv + kv * V) : u32x4{0, 0, 0, 0};
  }
  if constexpr (BIAS) bias_build<NT, DH>(bvec, bias, bias_load(bias, h, H));
  floatx4 adk[DH / 16], adv[DH / 16];
#pragma unroll
  for (int t = 0; t < DH / 16; ++t) adk[t] = adv[t] = floatx4{0.f, 0.f, 0.f, 0.f};

  for (int q0 = (k0 / BQ) * BQ; q0 < S; q0 += BQ) {
    __syncthreads();
    stage_kmajor<T, BQ, DKV, NT>(sQ, Qp + (int64_t)q0 * in.ldq, in.ldq, S - q0);
    stage_kmajor<T, BQ, DKV, NT>(sdO, dOp + (int64_t)q0 * d, d, S - q0);
    stage_mnmajor<T, DH, BQ / V, NT>(sQt, Qp + (int64_t)q0 * in.ldq, in.ldq, S - q0, typename AccPerm<T>::type());
    stage_mnmajor<T, DH, BQ / V, NT>(sdOt, dOp + (int64_t)q0 * d, d, S - q0, typename AccPerm<T>::type());
    if (threadIdx.x < BQ) {
      const int q = q0 + threadIdx.x;
      sL[threadIdx.x] = (q < S) ? query_lse<BIAS>(Lp[q]) : 0.f;
      sD[threadIdx.x] = (q < S) ? Dp[q] : 0.f;
    }
    __syncthreads();
    floatx4 P[BQ / 16], dS[BQ / 16];
#pragma unroll
    for (int qt = 0; qt < BQ / 16; ++qt) {
      floatx4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < QSTEPS; ++st) {
        mma_step<T>(s, lds_frag<BQ>(sQ, st, qt * 16), kf[st]);
        mma_step<T>(dp, lds_frag<BQ>(sdO, st, qt * 16), vf[st]);
      }
      const uint32_t bits = DROP ? drop_col4(drop, bh, q0 + qt * 16 + 4 * (l >> 4), key) : 0xfu;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int qi = qt * 16 + 4 * (l >> 4) + r;
        const int q = q0 + qi;
        const bool ok = (key <= q) && (q < S) && (key < S);
        const float bv = BIAS ? bvec[BIAS_FRONT + min(max(q - key, 0), bias.max_distance)] : 0.f;
        const float p = ok ? exp2f((BIAS ? s[r] + bv : s[r]) * scale_log2 - sL[qi]) : 0.f;
        // dropout M = keep * scale: dV takes P M, dP = (dO V^T) M
        const float mk = DROP ? (((bits >> r) & 1) ? drop.scale : 0.f) : 1.f;
        P[qt][r] = p * mk;
        dS[qt][r] = p * (dp[r] * mk - sD[qi]);
      }
    }
#pragma unroll
    for (int st = 0; st < RSTEPS; ++st) {
      const u32x4 pf = acc_to_frag<T>(P, st), sf = acc_to_frag<T>(dS, st);
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) {
        mma_step<T>(adv[t], lds_frag<DH>(sdOt, st, t * 16), pf);
        mma_step<T>(adk[t], lds_frag<DH>(sQt, st, t * 16), sf);
      }
    }
  }
  if (key < S) {
    T* dk = grad.k + ((int64_t)b * S + key) * grad.ldk + h * DH;
    T* dv = grad.v + ((int64_t)b * S + key) * grad.ldv + h * DH;
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) {
      const int c = t * 16 + 4 * (l >> 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        dk[c + r] = from_f32<T>(adk[t][r] * scale);
        dv[c + r] = from_f32<T>(adv[t][r]);
      }
    }
  }
}

template <typename T, int DH, bool DROP, bool BIAS>
__device__ __forceinline__ void dq_body(u32x4* tiles, float* bvec, int yb, const QkvView<T>& in, const T* dO,
                                        const float* lse2, const float* Dsum, const GradView<T>& grad, int S, int H, int d,
                                        float scale_log2, float scale, const DropArgs& drop, const BiasArgs& bias) {
  constexpr int V = Vec<T>::V;
  constexpr int BQ = 64;
  constexpr int DKV = DH / V;
  constexpr int QSTEPS = DH / (4 * V);
  constexpr int PSTEPS = BKV / (4 * V);
  u32x4* sK = tiles;
  u32x4* sV = sK + DKV * BKV;
  u32x4* sKt = sV + DKV * BKV;

  const int nqb = (S + BQ - 1) / BQ;
  const int qb = nqb - 1 - yb;
  const int bh = blockIdx.y, b = bh / H, h = bh % H;
  const int w = threadIdx.x >> 6, l = lane_id();
  const T* Qp = in.q + (int64_t)b * S * in.ldq + h * DH;
  const T* Kp = in.k + (int64_t)b * S * in.ldk + h * DH;
  const T* Vp = in.v + (int64_t)b * S * in.ldv + h * DH;
  const T* dOp = dO + (int64_t)b * S * d + h * DH;
  const int q0 = qb * BQ;
  const int qrow = q0 + 16 * w + (l & 15);
  const bool qok = qrow < S;
  const float lq = qok ? query_lse<BIAS>(lse2[(int64_t)bh * S + qrow]) : 0.f;
  const float Dq = qok ? Dsum[(int64_t)bh * S + qrow] : 0.f;

  u32x4 qf[QSTEPS], gf[QSTEPS];
#pragma unroll
  for (int s = 0; s < QSTEPS; ++s) {
    const int kv = s * 4 + (l >> 4);
    qf[s] = qok ? ld16(Qp + (int64_t)qrow * in.ldq + kv * V) : u32x4{0, 0, 0, 0};
    gf[s] = qok ? ld16(dOp + (int64_t)qrow * d + kv * V) : u32x4{0, 0, 0, 0};
  }
  DiagSums<1> diag;
  if constexpr (BIAS) {
    const int qw0 = q0 + 16 * w, nrow = (S + 15) / 16;
    diag.init(bvec + bias_len(bias.max_distance) + 2 * bias.n_buckets,
              bias.part != nullptr && qw0 < S ? bias.part + (((int64_t)h * bias.batch + b) * nrow + qw0 / 16) * (bias.max_distance + 1) : nullptr,
              bias.max_distance);
    bias_build<NT, DH>(bvec, bias, bias_load(bias, h, H));
  }
  floatx4 adq[DH / 16];
#pragma unroll
  for (int t = 0; t < DH / 16; ++t) adq[t] = floatx4{0.f, 0.f, 0.f, 0.f};

  const int last_kb = min((q0 + BQ - 1) / BKV, (S - 1) / BKV);
  for (int kb = 0; kb <= last_kb; ++kb) {
    const int k0 = kb * BKV;
    __syncthreads();
    stage_kmajor<T, BKV, DKV, NT>(sK, Kp + (int64_t)k0 * in.ldk, in.ldk, S - k0);
    stage_kmajor<T, BKV, DKV, NT>(sV, Vp + (int64_t)k0 * in.ldv, in.ldv, S - k0);
    stage_mnmajor<T, DH, BKV / V, NT>(sKt, Kp + (int64_t)k0 * in.ldk, in.ldk, S - k0, typename AccPerm<T>::type());
    __syncthreads();
    floatx4 dS[BKV / 16];
#pragma unroll
    for (int kt = 0; kt < BKV / 16; ++kt) {
      floatx4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < QSTEPS; ++st) {
        mma_step<T>(s, lds_frag<BKV>(sK, st, kt * 16), qf[st]);
        mma_step<T>(dp, lds_frag<BKV>(sV, st, kt * 16), gf[st]);
      }
      const uint32_t bits = DROP ? drop_row4(drop, bh, qrow, k0 + kt * 16 + 4 * (l >> 4)) : 0xfu;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int key = k0 + kt * 16 + 4 * (l >> 4) + r;
        const bool ok = qok && (key <= qrow) && (key < S);
        const float bv = BIAS ? bvec[BIAS_FRONT + min(max(qrow - key, 0), bias.max_distance)] : 0.f;
        const float p = ok ? exp2f((BIAS ? s[r] + bv : s[r]) * scale_log2 - lq) : 0.f;
        const float mk = DROP ? (((bits >> r) & 1) ? drop.scale : 0.f) : 1.f;
        dS[kt][r] = p * (dp[r] * mk - Dq);
      }
    }
    if constexpr (BIAS) {
      if (diag.out != nullptr) {   // uniform in a wavefront
        float acc[4][4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[3 - kt][r] = dS[kt][r];
        diag.block(q0 + 16 * w - k0, acc);
      }
    }
#pragma unroll
    for (int st = 0; st < PSTEPS; ++st) {
      const u32x4 sf = acc_to_frag<T>(dS, st);
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) mma_step<T>(adq[t], lds_frag<DH>(sKt, st, t * 16), sf);
    }
  }
  if (qok) {
    T* dq = grad.q + ((int64_t)b * S + qrow) * grad.ldq + h * DH;
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) {
      const int c = t * 16 + 4 * (l >> 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) dq[c + r] = from_f32<T>(adq[t][r] * scale);
    }
  }
  if constexpr (BIAS) {
    if (diag.out != nullptr) diag.finish(q0 + 16 * w - last_kb * BKV);
  }
}

// dK/dV of key block x below nkb, then dQ (largest queries first): one launch, so that both
// kinds share the CUs (2 x 512 tokens, 8 heads of 64: 147 us a pass as two launches, 87 as
// one) and one launch less where that counts (4 x 64 tokens, 4 heads of 32: 20 -> 17 us).
template <typename T, int DH, bool DROP, bool BIAS>
__global__ void __launch_bounds__(NT, 2) attn_bwd_kernel(QkvView<T> in, const T* dO, const float* lse2, const float* Dsum,
                                                      GradView<T> grad, int S, int H, int d, float scale_log2, float scale,
                                                      DropArgs drop, int nkb, BiasArgs bias) {
  __shared__ u32x4 tiles[BwdTiles<T, DH>::SLOTS];
  extern __shared__ float bvec[];
  if ((int)blockIdx.x < nkb)
    dkdv_body<T, DH, DROP, BIAS>(tiles, bvec, blockIdx.x, in, dO, lse2, Dsum, grad, S, H, d, scale_log2, scale, drop, bias);
  else
    dq_body<T, DH, DROP, BIAS>(tiles, bvec, blockIdx.x - nkb, in, dO, lse2, Dsum, grad, S, H, d, scale_log2, scale, drop, bias);
}

// ---------------------------------------------------------------------------------------
// Backward, bf16. A pre-pass writes (lse2, D) pairs per query into a buffer
// padded to 64 queries per head, so the workgroups can copy them with the
// blocks. Two kinds of workgroup, in one launch, then recompute P from q, k and
// lse2 (no atomics):
//   dK/dV  per 64 * SUB keys of a wavefront (K and V fragments in registers),
//          streaming 64-query blocks of Q, dO and their pairs through the ring:
//          S = Q K^T and dP = dO V^T with the key in the lane, then
//          dV^T += dO^T P and dK^T += Q^T dS, dO^T and Q^T by transpose reads;
//   dQ     per 64 * SUB queries (Q and dO fragments in registers), streaming
//          64-key blocks of K and V: S^T, dP^T with the query in the lane, then
//          dQ^T += K^T dS^T, K^T by transpose reads.
// head_dim 64: workgroups of 4 wavefronts of 32 rows, two per CU. Each has its
// own barrier, so the two wavefronts of a SIMD drift apart and one's softmax
// VALU work overlaps the other's MFMAs (one workgroup of 8 wavefronts per CU
// keeps them in step: 9% slower for dK/dV, 4% for dQ). 128: 8 of 16 rows;
// 32: 4 of 64 rows.
// SMALL: 4 wavefronts of 16 rows, for grids that would leave CUs idle.
template <int DH, bool SMALL = false> struct BwdRing {
  static constexpr int CPR = DH / 8, KST = DH / 32;
  static constexpr int SUB = SMALL ? 1 : DH == 32 ? 4 : (DH == 64 ? 2 : 1), WAVES = DH == 128 && !SMALL ? 8 : 4,
                       NTB = 64 * WAVES;
  static constexpr int OCC = DH == 32 && !SMALL ? 1 : 2;   // wavefronts per SIMD the register budget must allow
  static constexpr int WR = 16 * SUB, BR = WAVES * WR;
  static constexpr int NS = 4;
  static constexpr int BLK = 64 * CPR;
  static constexpr int PAIR_SLOTS = 32;            // 64 (lse2, D) pairs
  static constexpr int STAGE = 2 * BLK + PAIR_SLOTS;
  static constexpr int L = 2 * BLK / NTB;          // block loads per thread per stage (wave 0 adds the pairs)
};

// (lse2, D) pairs: LPR threads per (token, head) row, PAIR_ROWS consecutive
// rows per thread group with all their loads issued first.
constexpr int PAIR_ROWS = 2;
template <int DH>
__global__ void __launch_bounds__(NT) attn_pairs_kernel(const bf16* o, const bf16* dO, const float* lse2, float* pairs,
                                                         int S, int S_pad, int H, int d, int64_t rows) {
  constexpr int LPR = DH / 8;
  const int64_t gid = (int64_t)blockIdx.x * NT + threadIdx.x;
  const int64_t row0 = gid / LPR * PAIR_ROWS;  // row = token * H + h
  const int part = gid % LPR;
  u32x4 a[PAIR_ROWS], g[PAIR_ROWS];
#pragma unroll
  for (int i = 0; i < PAIR_ROWS; ++i) {
    const int64_t row = row0 + i;
    const int64_t off = (row / H) * d + (row % H) * DH + part * 8;
    a[i] = row < rows ? ld16(o + off) : u32x4{0, 0, 0, 0};
    g[i] = row < rows ? ld16(dO + off) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < PAIR_ROWS; ++i) {
    const int64_t row = row0 + i;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += vget<bf16>(a[i], j) * vget<bf16>(g[i], j);
#pragma unroll
    for (int m = LPR / 2; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);
    if (row < rows && part == 0) {
      const int64_t tok = row / H, bq = tok / S, q = tok % S;
      const int64_t bh = bq * H + row % H;
      pairs[(bh * S_pad + q) * 2] = lse2[bh * S + q];
      pairs[(bh * S_pad + q) * 2 + 1] = sum;
    }
  }
  // queries S .. S_pad - 1 of every head: zeros, so that masked products (p = 0) stay finite
  const int npad = S_pad - S;
  const int64_t heads = rows / S;
  if (npad > 0 && gid < heads * npad) {
    const int64_t bh = gid / npad, q = S + gid % npad;
    pairs[(bh * S_pad + q) * 2] = 0.f;
    pairs[(bh * S_pad + q) * 2 + 1] = 0.f;
  }
}

// The same with a bias: D as the diagonal of the products dO o^T, one wavefront per 16 queries
// of a head, in the steps in which the backward forms dP = dO V^T. A query that sees one key
// has o = v; the two sums are then the same float and its dS is zero, as it has to be. D by
// another order leaves the rounding of a sum (1e-7 of |dO v|), which is all that a table's
// gradient holds where every query sees one key. bf16: (lse2, D) pairs, with +inf for the lse2
// of a query that sees none, and zeros behind the sequence; fp32: D alone. A pass is no longer
// for it: 8 x 1024 tokens, 16 heads of 64: 114.6 us, 115.0 with the kernel above; 2 x 777, 3 heads
// of 64: 32.6, 33.5. Without a bias the kernels above stay, and with them their bits.
template <typename T, int DH>
__global__ void __launch_bounds__(NT) attn_bias_dsum_kernel(const T* o, const T* dO, const float* lse2, float* out, int S,
                                                             int S_pad, int H, int d, int64_t tiles) {
  constexpr int V = Vec<T>::V, STEPS = DH / (4 * V);
  const int l = lane_id(), g = l >> 4, c = l & 15;
  const int64_t tile = (int64_t)blockIdx.x * (NT / 64) + (threadIdx.x >> 6);   // (sequence, 16 queries, head)
  if (tile >= tiles) return;
  const int h = tile % H, q = (int)(tile / H % (S_pad / 16)) * 16 + c;
  const int64_t b = tile / H / (S_pad / 16), bh = b * H + h;
  const bool ok = q < S;
  const int64_t off = (b * S + q) * d + h * DH + g * V;
  u32x4 x[STEPS], y[STEPS];
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    x[s] = ok ? ld16(dO + off + s * 4 * V) : u32x4{0, 0, 0, 0};
    y[s] = ok ? ld16(o + off + s * 4 * V) : u32x4{0, 0, 0, 0};
  }
  const float lq = ok ? lse2[bh * S + q] : 0.f;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < STEPS; ++s) mma_step<T>(acc, x[s], y[s]);
  if ((c >> 2) != g) return;   // lane (g, c) holds rows 4 g + r of column c
  const float D = (c & 2) ? ((c & 1) ? acc[3] : acc[2]) : ((c & 1) ? acc[1] : acc[0]);
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<float2*>(out + (bh * S_pad + q) * 2) = make_float2(query_lse<true>(lq), D);
  else if (ok)
    out[bh * S + q] = D;
}

// Column sums of the gradient tiles a workgroup holds, for the bias gradient of
// the qkv projection: lane l holds columns 4 (l >> 4) + r of 16-column tile t,
// for token l & 15; the 16 lanes of equal l >> 4 (one DPP row) are summed with
// row moves, the waves through LDS (red: WAVES * NCOL floats, free for this
// use), and each column goes out as one atomic add to col(c), unless that is null.
template <int WAVES, int NCOL, class Col>
__device__ __forceinline__ void colsum_tiles(float (&v)[NCOL / 16][4], float* red, Col col) {
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4;
#pragma unroll
  for (int t = 0; t < NCOL / 16; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) v[t][r] = row_sum16(v[t][r]);
  if ((l & 15) == 0) {
#pragma unroll
    for (int t = 0; t < NCOL / 16; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[w * NCOL + t * 16 + 4 * g + r] = v[t][r];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < NCOL; c += WAVES * 64) {
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < WAVES; ++u) sum += red[u * NCOL + c];
    float* to = col(c);
    if (to != nullptr) atomicAdd(to, sum);
  }
}

// dK/dV of key block kb (ring: NS * STAGE slots of LDS)
template <int DH, bool DROP, bool SMALL, bool BIAS>
__device__ __forceinline__ void dkdv_ring_body(u32x4* ring, float* bvec, int kb, const QkvView<bf16>& in, const bf16* dO,
                                               const float* pairs, const GradView<bf16>& grad, int S, int S_pad, int H,
                                               int d, float scale_log2, float scale, const DropArgs& drop,
                                               const BiasArgs& bias) {
  using C = BwdRing<DH, SMALL>;
  constexpr int SUB = C::SUB, KST = C::KST, NS = C::NS, CPR = C::CPR;
  static_assert(NS * C::STAGE * 4 >= C::WAVES * 2 * DH, "LDS for the column sums");
  const int bh = blockIdx.x, b = bh / H, h = bh % H;
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4;
  const int wu = __builtin_amdgcn_readfirstlane(w);
  const bf16* Qp = in.q + (int64_t)b * S * in.ldq + h * DH;
  const bf16* Kp = in.k + (int64_t)b * S * in.ldk + h * DH;
  const bf16* Vp = in.v + (int64_t)b * S * in.ldv + h * DH;
  const bf16* dOp = dO + (int64_t)b * S * d + h * DH;
  const float* Pp = pairs + (int64_t)bh * S_pad * 2;
  const uint32_t ring_lds = lds_addr(ring);
  const int k0 = kb * C::BR, kw0 = k0 + w * C::WR;
  const int nqb = (S + 63) / 64, qb_first = k0 / 64, njobs = nqb - qb_first;
  const int my_first = (kw0 < S) ? kw0 / 64 : nqb;

  u32x4 kf[SUB][KST], vf[SUB][KST];
#pragma unroll
  for (int ks = 0; ks < SUB; ++ks) {
    const int key = kw0 + 16 * ks + (l & 15);
#pragma unroll
    for (int st = 0; st < KST; ++st) {
      kf[ks][st] = (key < S) ? ld16(Kp + (int64_t)key * in.ldk + st * 32 + 8 * g) : u32x4{0, 0, 0, 0};
      vf[ks][st] = (key < S) ? ld16(Vp + (int64_t)key * in.ldv + st * 32 + 8 * g) : u32x4{0, 0, 0, 0};
    }
  }
  floatx4 adk[SUB][DH / 16], adv[SUB][DH / 16];
#pragma unroll
  for (int ks = 0; ks < SUB; ++ks)
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) adk[ks][t] = adv[ks][t] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto fill = [&](int j) {
    const uint32_t st = ring_lds + (uint32_t)((j % NS) * C::STAGE * 16);
    const int q0 = (qb_first + j) * 64;
    blk_fill<CPR, C::NTB>(Qp + (int64_t)q0 * in.ldq, in.ldq, S - q0, st, wu, l);
    blk_fill<CPR, C::NTB>(dOp + (int64_t)q0 * d, d, S - q0, st + C::BLK * 16, wu, l);
    if (wu == 0 && l < C::PAIR_SLOTS) dma16(Pp + (int64_t)q0 * 2 + l * 4, st + 2 * C::BLK * 16);
  };
  BiasEntry entry{};
  if constexpr (BIAS) entry = bias_load(bias, h, H);
#pragma unroll
  for (int t = 0; t < NS - 1; ++t)
    if (t < njobs) fill(t);
  wait_vmcnt_all();   // kf and vf known complete: no vmcnt(0) inside the loop
  if constexpr (BIAS) bias_build<C::NTB, DH>(bvec, bias, entry);
  for (int j = 0; j < njobs; ++j) {
    wait_loads<C::L, NS - 2>(min(njobs - 1, j + NS - 2) - j);
    wait_lds_reads();
    barrier_no_fence();
    if (j + NS - 1 < njobs) fill(j + NS - 1);
    const int qb = qb_first + j;
    if (qb < my_first) continue;
    const u32x4* sQ = ring + (j % NS) * C::STAGE;
    const u32x4* sdO = sQ + C::BLK;
    const float* sP = reinterpret_cast<const float*>(sQ + 2 * C::BLK);
    const int q0 = qb * 64;
    const bool edge = (q0 < kw0 + C::WR - 1) || (q0 + 64 > S) || (kw0 + C::WR > S);
    // the bias of query 16 t + 4 g + r and key 16 ks + l % 16 of these: bp[16 (t - ks) + r]
    const float* bp = BIAS ? bvec + BIAS_FRONT + min(q0 - kw0, bias.max_distance + C::WR - 1) + 4 * g - (l & 15) : nullptr;
#pragma unroll
    for (int s = 0; s < 2; ++s) {   // 32 queries: tiles 2s and 2s + 1
      floatx4 sc[SUB][2], dp[SUB][2];
      floatx4 bv[SUB + 1];   // bias of the tiles' distances 2 s + u - ks
      if constexpr (BIAS) {
#pragma unroll
        for (int i = 0; i <= SUB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) bv[i][r] = bp[16 * (2 * s + i - SUB + 1) + r];
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 qfr[KST], gfr[KST];
#pragma unroll
        for (int st = 0; st < KST; ++st) {
          qfr[st] = blk_frag<CPR>(sQ, st, (2 * s + u) * 16);
          gfr[st] = blk_frag<CPR>(sdO, st, (2 * s + u) * 16);
        }
#pragma unroll
        for (int ks = 0; ks < SUB; ++ks) {
          sc[ks][u] = dp[ks][u] = floatx4{0.f, 0.f, 0.f, 0.f};
          if constexpr (BIAS) sc[ks][u] = bv[u - ks + SUB - 1];
#pragma unroll
          for (int st = 0; st < KST; ++st) {
            mma_step<bf16>(sc[ks][u], qfr[st], kf[ks][st]);
            mma_step<bf16>(dp[ks][u], gfr[st], vf[ks][st]);
          }
        }
      }
      // P = 2^(s * scale * log2 e - lse2), dS = P (dP - D); masked entries get P = 0.
      // Dropout M = keep * scale: dV takes P M, and dP = (dO V^T) M.
      uint32_t dbits[2][SUB];
      if constexpr (DROP) drop_col4_quad<SUB>(drop, bh, q0 + 32 * s, kw0, dbits);
      auto softmax = [&](auto masked) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int qi = (2 * s + u) * 16 + 4 * g + r;
            const float lq = sP[2 * qi], Dq = sP[2 * qi + 1];
#pragma unroll
            for (int ks = 0; ks < SUB; ++ks) {
              float x = fmaf(sc[ks][u][r], scale_log2, -lq);
              if constexpr (decltype(masked)::value) {
                const int key = kw0 + 16 * ks + (l & 15);
                x = (key <= q0 + qi && q0 + qi < S && key < S) ? x : -INFINITY;
              }
              const float p = fast_exp2(x);
              if constexpr (DROP) {
                const float mk = ((dbits[u][ks] >> r) & 1) ? drop.scale : 0.f;
                sc[ks][u][r] = p * mk;
                dp[ks][u][r] = p * (dp[ks][u][r] * mk - Dq);
              } else {
                sc[ks][u][r] = p;
                dp[ks][u][r] = p * (dp[ks][u][r] - Dq);
              }
            }
          }
      };
      if (edge) softmax(std::true_type());
      else softmax(std::false_type());
      u32x4 pfr[SUB], dsf[SUB];
#pragma unroll
      for (int ks = 0; ks < SUB; ++ks) {
        pfr[ks] = acc_to_frag<bf16>(sc[ks], 0);
        dsf[ks] = acc_to_frag<bf16>(dp[ks], 0);
      }
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) {
        const u32x4 gt = blk_frag_tr<CPR>(sdO, s, t * 16), qt = blk_frag_tr<CPR>(sQ, s, t * 16);
#pragma unroll
        for (int ks = 0; ks < SUB; ++ks) {
          mma_step<bf16>(adv[ks][t], gt, pfr[ks]);
          mma_step<bf16>(adk[ks][t], qt, dsf[ks]);
        }
      }
    }
  }
#pragma unroll
  for (int ks = 0; ks < SUB; ++ks) {
    const int key = kw0 + 16 * ks + (l & 15);
    if (key < S) {
      bf16* dk = grad.k + ((int64_t)b * S + key) * grad.ldk + h * DH;
      bf16* dv = grad.v + ((int64_t)b * S + key) * grad.ldv + h * DH;
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) {
        *reinterpret_cast<u32x2*>(dk + t * 16 + 4 * g) =
            u32x2{pack_bf16x2(adk[ks][t][0] * scale, adk[ks][t][1] * scale),
                  pack_bf16x2(adk[ks][t][2] * scale, adk[ks][t][3] * scale)};
        *reinterpret_cast<u32x2*>(dv + t * 16 + 4 * g) =
            u32x2{pack_bf16x2(adv[ks][t][0], adv[ks][t][1]), pack_bf16x2(adv[ks][t][2], adv[ks][t][3])};
      }
    }
  }
  if (grad.sv != nullptr) {   // uniform: bias gradients += column sums of dK and dV over this workgroup's keys
    float v[2 * DH / 16][4];
#pragma unroll
    for (int t = 0; t < DH / 16; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float sk = 0.f, sv = 0.f;
#pragma unroll
        for (int ks = 0; ks < SUB; ++ks) {
          sk += adk[ks][t][r];
          sv += adv[ks][t][r];
        }
        v[t][r] = sk * scale;
        v[DH / 16 + t][r] = sv;
      }
    __syncthreads();   // every wave is done with the ring
    colsum_tiles<C::WAVES, 2 * DH>(v, reinterpret_cast<float*>(ring), [&](int c) -> float* {
      return c >= DH ? grad.sv + h * DH + c - DH : grad.sk != nullptr ? grad.sk + h * DH + c : nullptr;
    });
  }
}

// dQ of query block nqb - 1 - yb (ring: NS * 2 * BLK slots of LDS)
template <int DH, bool DROP, bool SMALL, bool BIAS>
__device__ __forceinline__ void dq_ring_body(u32x4* ring, float* bvec, int yb, const QkvView<bf16>& in, const bf16* dO,
                                             const float* pairs, const GradView<bf16>& grad, int S, int S_pad, int H,
                                             int d, float scale_log2, float scale, const DropArgs& drop,
                                             const BiasArgs& bias) {
  using C = BwdRing<DH, SMALL>;
  constexpr int SUB = C::SUB, KST = C::KST, NS = C::NS, CPR = C::CPR;
  static_assert(NS * 2 * C::BLK * 4 >= C::WAVES * DH, "LDS for the column sums");
  const int nqb = (S + C::BR - 1) / C::BR;
  const int qb = nqb - 1 - yb;                   // largest queries first: they see the most keys
  const int bh = blockIdx.x, b = bh / H, h = bh % H;
  const int w = threadIdx.x >> 6, l = lane_id(), g = l >> 4;
  const int wu = __builtin_amdgcn_readfirstlane(w);
  const bf16* Qp = in.q + (int64_t)b * S * in.ldq + h * DH;
  const bf16* Kp = in.k + (int64_t)b * S * in.ldk + h * DH;
  const bf16* Vp = in.v + (int64_t)b * S * in.ldv + h * DH;
  const bf16* dOp = dO + (int64_t)b * S * d + h * DH;
  const float* Pp = pairs + (int64_t)bh * S_pad * 2;
  const uint32_t ring_lds = lds_addr(ring);
  const int q0 = qb * C::BR, qw0 = q0 + w * C::WR;
  const int nkb = min((q0 + C::BR - 1) / BKV, (S - 1) / BKV) + 1;
  const int my_last = (qw0 < S) ? min((qw0 + C::WR - 1) / BKV, (S - 1) / BKV) : -1;

  u32x4 qf[SUB][KST], gf[SUB][KST];
  float lq[SUB], Dq[SUB];
#pragma unroll
  for (int qs = 0; qs < SUB; ++qs) {
    const int q = qw0 + 16 * qs + (l & 15);
    const bool ok = q < S;
#pragma unroll
    for (int st = 0; st < KST; ++st) {
      qf[qs][st] = ok ? ld16(Qp + (int64_t)q * in.ldq + st * 32 + 8 * g) : u32x4{0, 0, 0, 0};
      gf[qs][st] = ok ? ld16(dOp + (int64_t)q * d + st * 32 + 8 * g) : u32x4{0, 0, 0, 0};
    }
    lq[qs] = ok ? Pp[2 * q] : 0.f;
    Dq[qs] = ok ? Pp[2 * q + 1] : 0.f;
  }
  floatx4 adq[SUB][DH / 16];
#pragma unroll
  for (int qs = 0; qs < SUB; ++qs)
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) adq[qs][t] = floatx4{0.f, 0.f, 0.f, 0.f};

  auto fill = [&](int kb) {
    const uint32_t st = ring_lds + (uint32_t)((kb % NS) * 2 * C::BLK * 16);
    const int k0 = kb * BKV;
    blk_fill<CPR, C::NTB>(Kp + (int64_t)k0 * in.ldk, in.ldk, S - k0, st, wu, l);
    blk_fill<CPR, C::NTB>(Vp + (int64_t)k0 * in.ldv, in.ldv, S - k0, st + C::BLK * 16, wu, l);
  };
  BiasEntry entry{};
  if constexpr (BIAS) entry = bias_load(bias, h, H);
#pragma unroll
  for (int t = 0; t < NS - 1; ++t)
    if (t < nkb) fill(t);
  wait_vmcnt_all();   // qf, gf, lq and Dq known complete: no vmcnt(0) inside the loop
  DiagSums<SUB> sums;
  float far_sum[4] = {0.f, 0.f, 0.f, 0.f};   // of dS over blocks beyond max_distance
  if constexpr (BIAS) {
    const int nrow = (S + C::WR - 1) / C::WR;
    sums.init(bvec + bias_len(bias.max_distance) + 2 * bias.n_buckets,
              bias.part != nullptr && qw0 < S ? bias.part + (((int64_t)h * bias.batch + b) * nrow + qw0 / C::WR) * (bias.max_distance + 1) : nullptr,
              bias.max_distance);
    bias_build<C::NTB, DH>(bvec, bias, entry);
  }
  for (int kb = 0; kb < nkb; ++kb) {
    wait_loads<C::L, NS - 2>(min(nkb - 1, kb + NS - 2) - kb);
    wait_lds_reads();
    barrier_no_fence();
    if (kb + NS - 1 < nkb) fill(kb + NS - 1);
    if (kb > my_last) continue;
    const u32x4* sK = ring + (kb % NS) * 2 * C::BLK;
    const u32x4* sV = sK + C::BLK;
    const int k0 = kb * BKV;
    const bool edge = (k0 + BKV - 1 > qw0) || (k0 + BKV > S) || (qw0 + C::WR > S);
    const bool near = !BIAS || edge || qw0 - k0 - (BKV - 1) < bias.max_distance;   // dS goes to more than one distance
    const float* bp = BIAS ? bvec + BIAS_FRONT + min(qw0 - k0, bias.max_distance + 63) + (l & 15) - 4 * g : nullptr;
    float diag[SUB + 3][4];
    if constexpr (BIAS) {
#pragma unroll
      for (int i = 0; i < SUB + 3; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) diag[i][r] = 0.f;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {   // 32 keys: tiles 2s and 2s + 1
      floatx4 sc[SUB][2], dp[SUB][2];
      floatx4 bv[SUB + 1];   // bias of the tiles' distances qs - 2 s - u
      if constexpr (BIAS) {
#pragma unroll
        for (int i = 0; i <= SUB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) bv[i][r] = bp[16 * (i - 1 - 2 * s) - r];
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 kfr[KST], vfr[KST];
#pragma unroll
        for (int st = 0; st < KST; ++st) {
          kfr[st] = blk_frag<CPR>(sK, st, (2 * s + u) * 16);
          vfr[st] = blk_frag<CPR>(sV, st, (2 * s + u) * 16);
        }
#pragma unroll
        for (int qs = 0; qs < SUB; ++qs) {
          sc[qs][u] = dp[qs][u] = floatx4{0.f, 0.f, 0.f, 0.f};
          if constexpr (BIAS) sc[qs][u] = bv[qs - u + 1];
#pragma unroll
          for (int st = 0; st < KST; ++st) {
            mma_step<bf16>(sc[qs][u], kfr[st], qf[qs][st]);
            mma_step<bf16>(dp[qs][u], vfr[st], gf[qs][st]);
          }
        }
      }
      auto softmax = [&](auto masked, auto is_far) {
        constexpr bool FAR = decltype(is_far)::value;
#pragma unroll
        for (int qs = 0; qs < SUB; ++qs) {
          const int q = qw0 + 16 * qs + (l & 15);
          uint32_t dbits[2] = {0xfu, 0xfu};   // dropout M = keep * scale on dP = dO V^T
          if constexpr (DROP) drop_row4_pair(drop, bh, q, k0 + 32 * s + 4 * g, k0 + 32 * s + 16 + 4 * g, dbits[0], dbits[1]);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint32_t bits = dbits[u];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float x = fmaf(sc[qs][u][r], scale_log2, -lq[qs]);
              if constexpr (decltype(masked)::value) {
                const int key = k0 + (2 * s + u) * 16 + 4 * g + r;
                x = (key <= q && key < S && q < S) ? x : -INFINITY;
              }
              const float p = fast_exp2(x);
              const float mk = DROP ? (((bits >> r) & 1) ? drop.scale : 0.f) : 1.f;
              dp[qs][u][r] = p * (dp[qs][u][r] * mk - Dq[qs]);
              if constexpr (BIAS && !FAR) diag[qs - 2 * s - u + 3][r] += dp[qs][u][r];
              if constexpr (FAR) far_sum[r] += dp[qs][u][r];
            }
          }
        }
      };
      if (edge) softmax(std::true_type(), std::false_type());
      else if (near) softmax(std::false_type(), std::false_type());
      else if constexpr (BIAS) softmax(std::false_type(), std::true_type());
      u32x4 dsf[SUB];
#pragma unroll
      for (int qs = 0; qs < SUB; ++qs) dsf[qs] = acc_to_frag<bf16>(dp[qs], 0);
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) {
        const u32x4 kt = blk_frag_tr<CPR>(sK, s, t * 16);
#pragma unroll
        for (int qs = 0; qs < SUB; ++qs) mma_step<bf16>(adq[qs][t], kt, dsf[qs]);
      }
    }
    if constexpr (BIAS) {
      if (near && sums.out != nullptr) sums.block(qw0 - k0, diag);
    }
  }
#pragma unroll
  for (int qs = 0; qs < SUB; ++qs) {
    const int q = qw0 + 16 * qs + (l & 15);
    if (q < S) {
      bf16* dq = grad.q + ((int64_t)b * S + q) * grad.ldq + h * DH;
#pragma unroll
      for (int t = 0; t < DH / 16; ++t)
        *reinterpret_cast<u32x2*>(dq + t * 16 + 4 * g) =
            u32x2{pack_bf16x2(adq[qs][t][0] * scale, adq[qs][t][1] * scale),
                  pack_bf16x2(adq[qs][t][2] * scale, adq[qs][t][3] * scale)};
    }
  }
  if constexpr (BIAS) {
    if (sums.out != nullptr) {
      sums.far += (far_sum[0] + far_sum[1]) + (far_sum[2] + far_sum[3]);
      sums.finish(qw0 - my_last * BKV);
    }
  }
  if (grad.sq != nullptr) {   // uniform: bias gradient += column sums of dQ over this workgroup's queries
    float v[DH / 16][4];
#pragma unroll
    for (int t = 0; t < DH / 16; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float sq = 0.f;
#pragma unroll
        for (int qs = 0; qs < SUB; ++qs) sq += adq[qs][t][r];
        v[t][r] = sq * scale;
      }
    __syncthreads();   // every wave is done with the ring
    colsum_tiles<C::WAVES, DH>(v, reinterpret_cast<float*>(ring), [&](int c) { return grad.sq + h * DH + c; });
  }
}

// The backward kernel: dK/dV and dQ in one launch (grid y below ny: dK/dV of key
// block y, smallest keys first; the rest: dQ, largest queries first), so that
// the tail of the dK/dV blocks overlaps the first dQ blocks and the two share
// CUs (7% faster than two launches at head dim 64).
template <int DH, bool DROP, bool SMALL, bool BIAS>
__global__ void __launch_bounds__((BwdRing<DH, SMALL>::NTB), (BwdRing<DH, SMALL>::OCC)) attn_bwd_ring_kernel(QkvView<bf16> in, const bf16* dO, const float* pairs,
                                                               GradView<bf16> grad, int S, int S_pad, int H, int d,
                                                               float scale_log2, float scale, DropArgs drop, int ny,
                                                               BiasArgs bias) {
  using C = BwdRing<DH, SMALL>;
  constexpr int SLOTS = C::STAGE > 2 * C::BLK ? C::NS * C::STAGE : C::NS * 2 * C::BLK;
  __shared__ u32x4 ring[SLOTS];
  extern __shared__ float bvec[];
  if ((int)blockIdx.y < ny)
    dkdv_ring_body<DH, DROP, SMALL, BIAS>(ring, bvec, blockIdx.y, in, dO, pairs, grad, S, S_pad, H, d, scale_log2, scale, drop,
                                          bias);
  else
    dq_ring_body<DH, DROP, SMALL, BIAS>(ring, bvec, blockIdx.y - ny, in, dO, pairs, grad, S, S_pad, H, d, scale_log2, scale,
                                        drop, bias);
}

// g_table[b][h] += the sum over sequences, wavefronts (wr queries each, `rows` of them) and
// the distances of bucket b of part [head][sequence][wavefront][max_distance + 1]. A
// wavefront has entries for the distances its queries reach. A workgroup takes the buckets
// of a head that begin at one of 16 distances (16 blockIdx.y and on): it sums their
// distances over the rows, side by side, then a wavefront adds up a bucket. All in a fixed
// order. Latency-bound: 16 loads a thread in flight, one round of them up to 512 rows. The
// columns are narrower than a cache line, so the workgroups of a head follow each other H
// apart: with 8 or 16 heads on one XCD, whose L2 then fetches a line once. 256 rows of 129 and
// 16 heads: 5.9 us (32 distances a workgroup 8.3; the workgroups of a head side by side
// 6.4), 512 rows of 257: 7.8 (11.0, 10.1), 512 of 513: 12.6 (11.5, 15.7).
constexpr int BS_NT = 512, BS_SPAN = 16;
__global__ void __launch_bounds__(BS_NT) attn_bias_sums_kernel(const float* __restrict__ part, int batch, int rows, int wr, int H,
                                                               const int32_t* __restrict__ bounds, int n_buckets,
                                                               int max_distance, float* g_table) {
  __shared__ float red[BS_NT];
  __shared__ float dist[MAX_DISTANCE + 1];
  __shared__ int begin[MAX_BUCKETS + 1];   // first distance of every bucket, then the end
  const int h = blockIdx.x, n = max_distance + 1, c = threadIdx.x & 63, rg = threadIdx.x >> 6;
  const int total = batch * rows;
  int b0 = 0, b1 = 0;   // the workgroup's buckets; every wavefront counts for itself
#pragma unroll
  for (int k = 0; k < MAX_BUCKETS / 64; ++k) {
    const int b = 64 * k + c;
    const int v = b == 0 ? 0 : b < n_buckets ? min(max(bounds[b], 0), n) : n;
    if (rg == 0) begin[b] = v;
    b0 += __popcll(__ballot(b < n_buckets && v < BS_SPAN * (int)blockIdx.y));
    b1 += __popcll(__ballot(b < n_buckets && v < BS_SPAN * ((int)blockIdx.y + 1)));
  }
  if (threadIdx.x == 0) begin[MAX_BUCKETS] = n;
  if (b0 >= b1) return;   // uniform
  float* g = g_table + (int64_t)(b0 + rg) * H + h;
  const float old = b0 + rg < b1 ? *g : 0.f;   // of the wavefront's first bucket
  __syncthreads();
  const int first = begin[b0], last = begin[b1];
  int cw = BS_SPAN;   // distances side by side: all of them if they are at most 128
  while (cw < last - first && cw < 128) cw *= 2;
  const int cc = threadIdx.x & (cw - 1), r0 = threadIdx.x / cw, step = BS_NT / cw;
  const float* mine = part + (int64_t)h * total * n;
  const int turn = step % rows;   // how far a step moves within the wavefronts of a sequence
  for (int d0 = first; d0 < last; d0 += cw) {
    const int d = min(d0 + cc, max_distance);
    float s = 0.f;
    int w = r0 % rows;
    for (int row0 = r0; row0 < total; row0 += 16 * step) {
      float v[16];   // loads first; entries beyond a wavefront's reach hold anything
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = mine[(int64_t)min(row0 + k * step, total - 1) * n + d];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        s += row0 + k * step < total && (d == max_distance || d < (w + 1) * wr) ? v[k] : 0.f;
        w += turn;
        if (w >= rows) w -= rows;
      }
    }
    if (cw <= 32) s += __shfl_xor(s, 32, 64);
    if (cw == 16) s += __shfl_xor(s, 16, 64);
    red[threadIdx.x] = s;
    __syncthreads();
    if (r0 == 0 && d0 + cc < n) {   // 8 row groups of 64 entries, or 4 of 128
      const int gs = max(cw, 64);
      s = 0.f;
#pragma unroll
      for (int q = 0; q < BS_NT / 64; ++q) s += q * gs < BS_NT ? red[(q * gs + cc) & (BS_NT - 1)] : 0.f;
      dist[d0 + cc] = s;
    }
    __syncthreads();
  }
  for (int b = b0 + rg; b < b1; b += BS_NT / 64) {
    float s = 0.f;
    for (int i = begin[b] + c; i < begin[b + 1]; i += 64) s += dist[i];
    s = wave_sum(s);
    if (c == 0) g_table[(int64_t)b * H + h] = s + (b == b0 + rg ? old : g_table[(int64_t)b * H + h]);
  }
}

// Whether workgroups of 64 rows (SMALL) fit the CUs about twice, so that the
// larger ones (2 to 4 times the rows) would not fill them: heads * ceil(S / 64)
// workgroups. Above that the larger ones share each K and V (Q and dO) fragment
// between more rows.
bool small_grid(int64_t heads, int S) { return heads * ((S + 63) / 64) <= 2 * cu_count(); }

template <typename T> QkvView<T> view(const AttnArgs& a) {
  return {reinterpret_cast<const T*>(a.q), reinterpret_cast<const T*>(a.k), reinterpret_cast<const T*>(a.v), a.ldq, a.ldk,
          a.ldv};
}
BiasArgs bias_args(const AttnArgs& a) { return {a.table, a.bounds, a.n_buckets, a.max_distance, a.mu, nullptr}; }
// bytes of LDS behind the tiles; diag: floats of the wavefronts' DiagRows
size_t bias_lds(const AttnArgs& a, int diag) {
  return a.table ? sizeof(float) * (size_t)bias_lds_floats(a.max_distance, a.n_buckets, diag) : 0;
}

template <typename T, int DH>
hipError_t fwd_launch(const AttnArgs& a, void* o, float* lse2, hipStream_t st) {
  const int mu = a.mu, S = a.S, H = a.H, d = H * DH;
  const float scale_log2 = LOG2E / sqrtf((float)DH);
  const size_t lds = bias_lds(a, 0);
  T* out = reinterpret_cast<T*>(o);
  auto launch = [&](auto bias) {
    constexpr bool B = decltype(bias)::value;
    if constexpr (sizeof(T) == 2) {
      auto go = [&](auto small) {
        constexpr bool SM = decltype(small)::value;
        using C = FwdRing<DH, SM>;
        dim3 grid(mu * H, (S + C::BQ - 1) / C::BQ);   // x fastest: every head's heaviest query block first
        auto k = a.drop.thr ? attn_fwd_ring_kernel<DH, true, SM, B> : attn_fwd_ring_kernel<DH, false, SM, B>;
        hipLaunchKernelGGL(k, grid, dim3(C::NTF), lds, st, view<T>(a), out, lse2, S, H, d, scale_log2, a.drop, bias_args(a));
      };
      if (small_grid(mu * H, S)) go(std::true_type{});
      else go(std::false_type{});
    } else {
      auto k = a.drop.thr ? attn_fwd_kernel<T, DH, true, B> : attn_fwd_kernel<T, DH, false, B>;
      hipLaunchKernelGGL(k, dim3((S + 63) / 64, mu * H), dim3(NT), lds, st, view<T>(a), out, lse2, S, H, d, scale_log2, a.drop,
                         bias_args(a));
    }
    return hipGetLastError();
  };
  return a.table ? launch(std::true_type{}) : launch(std::false_type{});
}

// Queries of a dQ wavefront.
int dq_wave_rows(const AttnArgs& a) {
  if (a.dt != DT_BF16 || small_grid(2 * (int64_t)a.mu * a.H, a.S)) return 16;
  return a.dh == 32 ? BwdRing<32>::WR : a.dh == 64 ? BwdRing<64>::WR : BwdRing<128>::WR;
}

template <typename T, int DH>
hipError_t bwd_launch(const AttnArgs& a, const AttnGrads& gr, const void* o, const void* dO, const float* lse2, float* ws,
                      float* bias_ws, hipStream_t st) {
  const int mu = a.mu, S = a.S, H = a.H, d = H * DH;
  const float scale = 1.f / sqrtf((float)DH);
  const float scale_log2 = LOG2E * scale;
  const T* g = reinterpret_cast<const T*>(dO);
  const GradView<T> grad{reinterpret_cast<T*>(gr.dq), reinterpret_cast<T*>(gr.dk), reinterpret_cast<T*>(gr.dv), gr.ldq, gr.ldk,
                         gr.ldv, gr.sum_q, gr.sum_k, gr.sum_v};
  BiasArgs ba = bias_args(a);
  if (a.table && gr.g_table) ba.part = bias_ws;
  const int64_t rows = (int64_t)mu * S * H;
  auto bias_dsum = [&](int S_pad) {
    const int64_t tiles = (int64_t)mu * H * (S_pad / 16);
    hipLaunchKernelGGL((attn_bias_dsum_kernel<T, DH>), dim3((unsigned)((tiles + NT / 64 - 1) / (NT / 64))), dim3(NT), 0, st,
                       reinterpret_cast<const T*>(o), g, lse2, ws, S, S_pad, H, d, tiles);
  };
  auto launch = [&](auto bias) {
    constexpr bool B = decltype(bias)::value;
    if constexpr (sizeof(T) == 2) {
      const int S_pad = (S + 63) / 64 * 64;
      if constexpr (!B) {
        const int64_t threads = (rows + PAIR_ROWS - 1) / PAIR_ROWS * (DH / 8);
        const int64_t pad_threads = (int64_t)mu * H * (S_pad - S);
        const int64_t grid_threads = threads > pad_threads ? threads : pad_threads;
        hipLaunchKernelGGL((attn_pairs_kernel<DH>), dim3((unsigned)((grid_threads + NT - 1) / NT)), dim3(NT), 0, st,
                           reinterpret_cast<const bf16*>(o), g, lse2, ws, S, S_pad, H, d, rows);
      } else {
        bias_dsum(S_pad);
      }
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      auto go = [&](auto small) {
        constexpr bool SM = decltype(small)::value;
        using C = BwdRing<DH, SM>;
        const int ny = (S + C::BR - 1) / C::BR;
        const dim3 grid(mu * H, 2 * ny);   // dK/dV blocks, then dQ blocks
        auto k = a.drop.thr ? attn_bwd_ring_kernel<DH, true, SM, B> : attn_bwd_ring_kernel<DH, false, SM, B>;
        hipLaunchKernelGGL(k, grid, dim3(C::NTB), bias_lds(a, C::WAVES * DiagRow<C::SUB>::FLOATS), st, view<T>(a), g, ws, grad, S, S_pad, H, d,
                           scale_log2, scale, a.drop, ny, ba);
      };
      if (small_grid(2 * (int64_t)mu * H, S)) go(std::true_type{});
      else go(std::false_type{});
      return hipGetLastError();
    } else {
      if constexpr (!B) {
        const int64_t threads = rows * (DH / Vec<T>::V);
        hipLaunchKernelGGL((attn_dsum_kernel<T, DH>), dim3((unsigned)((threads + NT - 1) / NT)), dim3(NT), 0, st,
                           reinterpret_cast<const T*>(o), g, ws, S, H, d, rows);
      } else {
        bias_dsum((S + 15) / 16 * 16);
      }
      hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      const int nkb = (S + BKV - 1) / BKV;
      auto k = a.drop.thr ? attn_bwd_kernel<T, DH, true, B> : attn_bwd_kernel<T, DH, false, B>;
      hipLaunchKernelGGL(k, dim3(2 * nkb, mu * H), dim3(NT), bias_lds(a, NT / 64 * DiagRow<1>::FLOATS), st, view<T>(a), g, lse2,
                         ws, grad, S, H, d, scale_log2, scale, a.drop, nkb, ba);
      e = hipGetLastError();
      // column sums: one pass where all three lie side by side
      if (e == hipSuccess && gr.sum_q != nullptr && gr.sum_k == gr.sum_q + d && gr.sum_v == gr.sum_k + d &&
          gr.ldk == gr.ldq && gr.ldv == gr.ldq && grad.k == grad.q + d && grad.v == grad.k + d)
        return colsum_acc(DT_F32, gr.dq, gr.ldq, mu * S, 3 * d, gr.sum_q, st);   // of this lambda
      if (e == hipSuccess && gr.sum_q != nullptr) e = colsum_acc(DT_F32, gr.dq, gr.ldq, mu * S, d, gr.sum_q, st);
      if (e == hipSuccess && gr.sum_k != nullptr) e = colsum_acc(DT_F32, gr.dk, gr.ldk, mu * S, d, gr.sum_k, st);
      if (e == hipSuccess && gr.sum_v != nullptr) e = colsum_acc(DT_F32, gr.dv, gr.ldv, mu * S, d, gr.sum_v, st);
      return e;
    }
  };
  hipError_t e = a.table ? launch(std::true_type{}) : launch(std::false_type{});
  if (e != hipSuccess || ba.part == nullptr) return e;
  const int wr = dq_wave_rows(a);
  hipLaunchKernelGGL(attn_bias_sums_kernel, dim3(H, a.max_distance / BS_SPAN + 1), dim3(BS_NT), 0, st, ba.part, mu, (S + wr - 1) / wr, wr, H,
                     a.bounds, a.n_buckets, a.max_distance, gr.g_table);
  return hipGetLastError();
}

bool attn_args_ok(const AttnArgs& a) {
  if (a.mu <= 0 || a.S <= 0 || a.H <= 0) return false;
  return !a.table || (a.bounds && a.n_buckets >= 1 && a.n_buckets <= MAX_BUCKETS && a.max_distance >= 1 &&
                      a.max_distance <= MAX_DISTANCE);
}

}  // namespace

// fp32 stops at head_dim 64: its backward's tiles take 65 KiB there and up to 11 KiB of bias, two
// workgroups to a CU's 160 KiB. At 128 the tiles alone would be 129 KiB, one workgroup of 4
// wavefronts to a CU.
hipError_t attn_fwd(const AttnArgs& a, void* o, float* lse2, hipStream_t st) {
  if (!attn_args_ok(a)) return hipErrorInvalidValue;
  if (a.dt == DT_BF16) {
    if (a.dh == 32) return fwd_launch<bf16, 32>(a, o, lse2, st);
    if (a.dh == 64) return fwd_launch<bf16, 64>(a, o, lse2, st);
    if (a.dh == 128) return fwd_launch<bf16, 128>(a, o, lse2, st);
    return hipErrorInvalidValue;
  }
  if (a.dh == 32) return fwd_launch<float, 32>(a, o, lse2, st);
  if (a.dh == 64) return fwd_launch<float, 64>(a, o, lse2, st);
  return hipErrorInvalidValue;
}

int64_t attn_bwd_workspace_floats(DType dt, int mu, int S, int H) {
  if (dt == DT_BF16) return 2 * (int64_t)mu * H * ((S + 63) / 64 * 64);
  return (int64_t)mu * H * S;
}
int64_t attn_bias_workspace_floats(const AttnArgs& a) {
  const int wr = dq_wave_rows(a);
  return (int64_t)a.mu * a.H * ((a.S + wr - 1) / wr) * (a.max_distance + 1);
}

hipError_t attn_bwd(const AttnArgs& a, const AttnGrads& g, const void* o, const void* dO, const float* lse2, float* ws,
                    float* bias_ws, hipStream_t st) {
  if (!attn_args_ok(a)) return hipErrorInvalidValue;
  if (a.dt == DT_BF16) {
    if (a.dh == 32) return bwd_launch<bf16, 32>(a, g, o, dO, lse2, ws, bias_ws, st);
    if (a.dh == 64) return bwd_launch<bf16, 64>(a, g, o, dO, lse2, ws, bias_ws, st);
    if (a.dh == 128) return bwd_launch<bf16, 128>(a, g, o, dO, lse2, ws, bias_ws, st);
    return hipErrorInvalidValue;
  }
  if (a.dh == 32) return bwd_launch<float, 32>(a, g, o, dO, lse2, ws, bias_ws, st);
  if (a.dh == 64) return bwd_launch<float, 64>(a, g, o, dO, lse2, ws, bias_ws, st);
  return hipErrorInvalidValue;
}

}  // namespace paci
