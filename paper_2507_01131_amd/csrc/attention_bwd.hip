// Backward of the attention block (attention.hip, launch_cp_edge_att), from
// the recomputed weights alpha.
//
// With Gz = grad_out W^T, U_t = D^T Gz[t] and V_s = A^T x[s] ([R, C] each), the
// products of an edge e = (s, t) per rank and head (C_h: the head's channels)
//   P_e[r, h] = sum over c in C_h of U_t[r, c] V_s[r, c]
// give both cotangents that the edge needs,
//   dalpha_e[h] = sum_r g_e[r] P_e[r, h],   dg_e[r] = sum_h alpha_e[h] P_e[r, h].
// k_att_dg forms P on 16-bit MFMA and keeps none of it: V^T of 32 ranks comes
// out with ranks in lanes and a head's channels in registers, where U_t^T of
// the destination already is, so the sum over channels stays in the lane.
// From dg on, the edge vectors' and radial weights' gradients are the layer's
// own (launch_bwd_dst with a.dg given).  The softmax and the logits' MLP,
//   da = alpha (dalpha - sum over the destination's edges of alpha dalpha),
//   dhid = LeakyReLU'(hid) (da w2^T),  hid = Pt[t] + Ps[s] + phi_e W1_phi,
// run in k_att_da, one wave a destination and one lane a hidden unit; what the
// hidden units owe to sources and destinations is summed per node and taken
// through W1 there (k_att_dps, k_att_dx0, k_att_dw1).  Every sum runs in a
// fixed order.
#include "common.hpp"
#include "kernels.h"
#include "sh_device.hpp"

namespace tdn {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kMaxF = 64, kMaxH = 8, kMaxRadial = 16;
constexpr float kLeaky = 0.2f;

__device__ __forceinline__ f32x16 mfma_f16(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                0);
}

// ---- the factors A and D [d, R] in the packed K order of
// launch_feature_layout_packed: [pk_blocks][rank tile][64 lanes] x 16 bytes,
// each rank's column in two fp16 parts of its values 2^-e, and 2^e [32 RT].
__global__ __launch_bounds__(256) void k_att_factors(int d, int R, int RT, const float* __restrict__ A,
                                                     const float* __restrict__ D, u32x4* __restrict__ ops,
                                                     float* __restrict__ scale) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * RT * kWave) return;
  const int which = i / (RT * kWave), rt = (i / kWave) % RT, lane = i & 63;
  const int h = lane >> 5, r = rt * kTile + (lane & 31), n = pk_rows(d), nb = pk_blocks(d);
  const float* F = which == 0 ? A : D;
  float mx = 0.f;
  if (r < R)
    for (int k = 0; k < d; ++k) mx = fmaxf(mx, fabsf(F[size_t(k) * R + r]));
  const int e = f16_split_exponent(mx);
  const float sc = ldexpf(1.f, -e);
  if (h == 0) scale[which * RT * kTile + r] = ldexpf(1.f, e);
  auto value = [&](int slot) {  // the factor's value of a lane's K slot
    const int part = slot / n, row = h * n + slot - part * n;
    const float v = part < 3 && row < d && r < R ? F[size_t(row) * R + r] * sc : 0.f;
    const float hi = float(_Float16(v));
    return part == 2 ? v - hi : hi;
  };
  u32x4* out = ops + size_t(which) * nb * RT * kWave;
  for (int b = 0; b < nb; ++b) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = pack_f16x2_rne(value(8 * b + 2 * k), value(8 * b + 2 * k + 1));
    out[(size_t(b) * RT + rt) * kWave + lane] = w;
  }
}

// ---- g_e [E, R] by sorted position: one thread a rank, harmonics and radial
// basis of 64 edges at a time in LDS.
constexpr int kGEdges = 64;
template <int L>
__global__ __launch_bounds__(256) void k_att_g(int E, int R, int nr, float sigma, const int32_t* __restrict__ perm,
                                               const float* __restrict__ edge_vec, const float* __restrict__ B,
                                               const float* __restrict__ Wr, float* __restrict__ g) {
  constexpr int d = (L + 1) * (L + 1);
  __shared__ float sY[kGEdges][d], sPhi[kGEdges][kMaxRadial];
  const int r = threadIdx.x, rc = min(r, R - 1);
  float b[d], w[kMaxRadial];
#pragma unroll
  for (int k = 0; k < d; ++k) b[k] = B[k * R + rc];
#pragma unroll
  for (int q = 0; q < kMaxRadial; ++q) w[q] = q < nr ? Wr[q * R + rc] : 0.f;
  const int e0 = blockIdx.x * kGEdges, n = min(kGEdges, E - e0);
  if (int(threadIdx.x) < n) {
    const int eid = perm[e0 + threadIdx.x];
    const float vx = edge_vec[3 * size_t(eid)], vy = edge_vec[3 * size_t(eid) + 1], vz = edge_vec[3 * size_t(eid) + 2];
    const float len = sqrtf(vx * vx + vy * vy + vz * vz), inv = 1.f / len;
    float Y[d];
    sh_unit_all<L>(vx * inv, vy * inv, vz * inv, Y);
#pragma unroll
    for (int k = 0; k < d; ++k) sY[threadIdx.x][k] = Y[k];
#pragma unroll
    for (int q = 0; q < kMaxRadial; ++q) sPhi[threadIdx.x][q] = radial_phi(len, q, sigma);
  }
  __syncthreads();
  if (r >= R) return;
  for (int e = 0; e < n; ++e) {
    float v = 0.f, rho = 0.f;
#pragma unroll
    for (int k = 0; k < d; ++k) v = fmaf(sY[e][k], b[k], v);
#pragma unroll
    for (int q = 0; q < kMaxRadial; ++q) rho = fmaf(sPhi[e][q], w[q], rho);
    g[size_t(e0 + e) * R + r] = v * rho;
  }
}

// ---- dg_e and, per rank tile, its share of dalpha_e
struct DgArgs {
  int E, C, R, RT, H, n_range;
  const int32_t *perm, *src, *dst;
  const uint32_t *xp, *gp;        // x and Gz in launch_feature_layout_packed's words
  const float *x_scale, *g_scale;  // their row scales
  const u32x4* ops;               // k_att_factors
  const float* f_scale;
  const float* g;                 // [E, R] by sorted position
  const float* alpha;             // [E, H] by sorted position
  float* dg;                      // [E, R]
  float* dal;                     // [RT, E, H]
};

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true);
  return v + __builtin_bit_cast(float, o);
}
// sum over the 32 lanes of a lane's half, in every lane of it
__device__ __forceinline__ float half_sum(float v) {
  v = dpp_add<0xB1>(v);   // quad_perm [1, 0, 3, 2]
  v = dpp_add<0x4E>(v);   // quad_perm [2, 3, 0, 1]
  v = dpp_add<0x141>(v);  // mirrored within 8 lanes
  v = dpp_add<0x140>(v);  // mirrored within 16 lanes
  return v + __shfl_xor(v, 16);
}
__device__ __forceinline__ float both_halves(float v) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// A wave takes one range of sorted edges and one tile of 32 ranks; the waves
// of a workgroup share a range as far as there are tiles, so that a source's
// words are read once from L2.
template <int L, int CT>
__global__ __launch_bounds__(256) void k_att_dg(DgArgs a) {
  constexpr int d = (L + 1) * (L + 1), n = pk_rows(d), nb = pk_blocks(d), n4 = n / 4, nt = n % 4;
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = xcd_remap(blockIdx.x, gridDim.x) * 4 + wave;
  const int range = item / a.RT, rt = item - range * a.RT;
  if (range >= a.n_range) return;
  const int e0 = int(int64_t(range) * a.E / a.n_range), e1 = int(int64_t(range + 1) * a.E / a.n_range);
  if (e0 >= e1) return;
  const int ct_n = a.C / kTile, per_head = ct_n / a.H, H = a.H, R = a.R;
  const int r = rt * kTile + l32;
  const float un = a.f_scale[r] * a.f_scale[a.RT * kTile + r];
  u32x4 Aop[nb];
#pragma unroll
  for (int b = 0; b < nb; ++b) Aop[b] = a.ops[(size_t(b) * a.RT + rt) * kWave + lane];
  const u32x4* Dop = a.ops + size_t(nb) * a.RT * kWave;
  // a node's words of one channel tile, as the K blocks of the contraction
  auto load_words = [&](const uint32_t* base, int node, int ct, uint32_t (&w)[n]) {
    const uint32_t* p = base + (size_t(node) * ct_n + ct) * 64 * n;
#pragma unroll
    for (int q = 0; q < n4; ++q) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p + q * 256 + 4 * lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * q + i] = v[i];
    }
#pragma unroll
    for (int i = 0; i < nt; ++i) w[4 * n4 + i] = p[n4 * 256 + nt * lane + i];
  };
  auto block = [&](const uint32_t (&w)[n], int b) {
    u32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = w[4 * b + k < n ? 4 * b + k : 4 * b + k - n];
    return v;
  };
  struct Rec {
    int src, dst;
    float sc;
  };
  auto load_batch = [&](int b0) {
    Rec rec{0, -1, 1.f};
    if (b0 + lane < e1) {
      const int eid = a.perm[b0 + lane];
      rec.src = a.src[eid];
      rec.dst = a.dst[eid];
      rec.sc = a.x_scale[rec.src] * a.g_scale[rec.dst];
    }
    return rec;
  };
  Rec cur = load_batch(e0), nxt = load_batch(e0 + kWave);
  int b0 = e0, t_cur = -1;
  f32x16 U[CT];
  uint32_t xw[n];
  load_words(a.xp, __builtin_amdgcn_readlane(cur.src, 0), 0, xw);
  for (int e = e0; e < e1; ++e) {
    const int j = e - b0;
    const int s = __builtin_amdgcn_readlane(cur.src, j), t = __builtin_amdgcn_readlane(cur.dst, j);
    const float sc = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, cur.sc), j)) * un;
    const int s_next = e + 1 >= e1 ? s
                                   : (j + 1 < kWave ? __builtin_amdgcn_readlane(cur.src, j + 1)
                                                    : __builtin_amdgcn_readlane(nxt.src, 0));
    if (t != t_cur) {
      t_cur = t;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        if (ct < ct_n) {
          uint32_t w[n];
          load_words(a.gp, t, ct, w);
          f32x16 acc = f32x16{};
#pragma unroll
          for (int b = 0; b < nb; ++b) acc = mfma_f16(block(w, b), Dop[(size_t(b) * a.RT + rt) * kWave + lane], acc);
          U[ct] = acc;
        }
    }
    const float ge = r < R ? a.g[size_t(e) * R + r] : 0.f;
    float p[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      p[ct] = 0.f;
      if (ct < ct_n) {
        uint32_t nw[n];
        const bool last = ct + 1 == ct_n;
        load_words(a.xp, last ? s_next : s, last ? 0 : ct + 1, nw);
        f32x16 V = f32x16{};
#pragma unroll
        for (int b = 0; b < nb; ++b) V = mfma_f16(block(xw, b), Aop[b], V);
#pragma unroll
        for (int v = 0; v < 16; ++v) p[ct] = fmaf(U[ct][v], V[v], p[ct]);
#pragma unroll
        for (int i = 0; i < n; ++i) xw[i] = nw[i];
      }
    }
    // per head: this lane's half of the channels, then both
    float dge = 0.f;
    for (int k = 0; k < H; ++k) {
      float P = 0.f;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        if (ct / per_head == k) P += p[ct];
      P = both_halves(P) * sc;
      dge = fmaf(a.alpha[size_t(e) * H + k], P, dge);
      const float da = half_sum(P * ge);
      if (lane == 0) a.dal[(size_t(rt) * a.E + e) * H + k] = da;
    }
    if (h == 0 && r < R) a.dg[size_t(e) * R + r] = dge;
    if (j + 1 == kWave) {
      cur = nxt;
      b0 += kWave;
      nxt = load_batch(b0 + kWave);
    }
  }
}

// ---- softmax and MLP: one wave a destination, one lane a hidden unit.  The
// workgroup's sums of grad w2 and of the radial rows of grad W1 go to partial
// [gridDim.x][n_radial + H][F].
constexpr int kDaWaves = 4;
__global__ __launch_bounds__(kDaWaves* kWave) void k_att_da(
    int N, int E, int C, int F, int H, int nr, int RT, float sigma, const int32_t* __restrict__ offsets,
    const int32_t* __restrict__ perm, const int32_t* __restrict__ src, const float* __restrict__ edge_vec,
    const float* __restrict__ Pt, const float* __restrict__ Ps, const float* __restrict__ W1,
    const float* __restrict__ w2, const float* __restrict__ alpha, const float* __restrict__ dal,
    float* __restrict__ dhid, float* __restrict__ dPt, float* __restrict__ grad_vec, float* __restrict__ partial) {
  __shared__ float s_da[kDaWaves][kWave][kMaxH];
  __shared__ float s_phi[kDaWaves][kWave][kMaxRadial], s_psi[kDaWaves][kWave][kMaxRadial];
  __shared__ float s_dl[kDaWaves][kWave];
  __shared__ int s_eid[kDaWaves][kWave], s_src[kDaWaves][kWave];
  __shared__ float s_red[kDaWaves][kWave];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool unit = lane < F;
  const float* Wphi = W1 + size_t(2 * C) * F;
  float wp[kMaxRadial], wo[kMaxH], gp[kMaxRadial], go[kMaxH];
#pragma unroll
  for (int q = 0; q < kMaxRadial; ++q) {
    wp[q] = unit && q < nr ? Wphi[q * F + lane] : 0.f;
    gp[q] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < kMaxH; ++k) {
    wo[k] = unit && k < H ? w2[lane * H + k] : 0.f;
    go[k] = 0.f;
  }
  // dalpha of sorted edge e and head k: the rank tiles' shares in order
  auto dalpha = [&](int e, int k) {
    float v = 0.f;
    for (int rt = 0; rt < RT; ++rt) v += dal[(size_t(rt) * E + e) * H + k];
    return v;
  };
  for (int t = blockIdx.x * kDaWaves + wv; t < N; t += gridDim.x * kDaWaves) {
    const int e0 = offsets[t], e1 = offsets[t + 1];
    float dpt = 0.f;
    if (e0 < e1) {
      float dot[kMaxH];
#pragma unroll
      for (int k = 0; k < kMaxH; ++k) {
        dot[k] = 0.f;
        if (k < H) {
          for (int e = e0 + lane; e < e1; e += kWave) dot[k] = fmaf(alpha[size_t(e) * H + k], dalpha(e, k), dot[k]);
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) dot[k] += __shfl_xor(dot[k], o);
        }
      }
      const float pt = unit ? Pt[size_t(t) * F + lane] : 0.f;
      for (int b = e0; b < e1; b += kWave) {
        const int cnt = min(kWave, e1 - b);
        // (one wave writes and reads its own rows: its LDS operations run in
        // order, the wave barriers keep the compiler from reordering them)
        __builtin_amdgcn_wave_barrier();
        float vx = 0.f, vy = 0.f, vz = 0.f, inv = 0.f;
        if (lane < cnt) {
          const int e = b + lane, eid = perm[e];
          s_eid[wv][lane] = eid;
          s_src[wv][lane] = src[eid];
#pragma unroll
          for (int k = 0; k < kMaxH; ++k)
            s_da[wv][lane][k] = k < H ? alpha[size_t(e) * H + k] * (dalpha(e, k) - dot[k]) : 0.f;
          vx = edge_vec[3 * size_t(eid)];
          vy = edge_vec[3 * size_t(eid) + 1];
          vz = edge_vec[3 * size_t(eid) + 2];
          const float len = sqrtf(vx * vx + vy * vy + vz * vz);
          inv = 1.f / len;
#pragma unroll
          for (int q = 0; q < kMaxRadial; ++q) {
            const float phi = q < nr ? radial_phi(len, q, sigma) : 0.f;
            s_phi[wv][lane][q] = phi;
            s_psi[wv][lane][q] = q < nr ? -radial_t(len, q, sigma) / sigma * phi : 0.f;
          }
        }
        __builtin_amdgcn_wave_barrier();
        float ps = unit ? Ps[size_t(s_src[wv][0]) * F + lane] : 0.f;
        for (int i = 0; i < cnt; ++i) {
          const float ps_next = unit && i + 1 < cnt ? Ps[size_t(s_src[wv][i + 1]) * F + lane] : 0.f;
          float hid = pt + ps, w = 0.f, dact = 0.f;
#pragma unroll
          for (int q = 0; q < kMaxRadial; ++q) {
            hid = fmaf(s_phi[wv][i][q], wp[q], hid);
            w = fmaf(s_psi[wv][i][q], wp[q], w);
          }
#pragma unroll
          for (int k = 0; k < kMaxH; ++k) dact = fmaf(s_da[wv][i][k], wo[k], dact);
          const float dh = hid > 0.f ? dact : kLeaky * dact, act = hid > 0.f ? hid : kLeaky * hid;
          dpt += dh;
#pragma unroll
          for (int q = 0; q < kMaxRadial; ++q) gp[q] = fmaf(s_phi[wv][i][q], dh, gp[q]);
#pragma unroll
          for (int k = 0; k < kMaxH; ++k) go[k] = fmaf(act, s_da[wv][i][k], go[k]);
          if (unit) dhid[size_t(s_eid[wv][i]) * F + lane] = dh;
          if (grad_vec) {
            const float dl = both_halves(half_sum(dh * w));
            if (lane == 0) s_dl[wv][i] = dl;
          }
          ps = ps_next;
        }
        __builtin_amdgcn_wave_barrier();
        if (grad_vec && lane < cnt) {
          float* gv = grad_vec + 3 * size_t(s_eid[wv][lane]);
          const float dl = s_dl[wv][lane] * inv;
          gv[0] += dl * vx;
          gv[1] += dl * vy;
          gv[2] += dl * vz;
        }
      }
    }
    if (unit) dPt[size_t(t) * F + lane] = dpt;
  }
  // the workgroup's sums over its waves, in order
#pragma unroll
  for (int i = 0; i < kMaxRadial + kMaxH; ++i) {
    const bool radial = i < kMaxRadial;
    const int k = radial ? i : i - kMaxRadial;
    if (k >= (radial ? nr : H)) continue;
    __syncthreads();
    s_red[wv][lane] = radial ? gp[radial ? k : 0] : go[radial ? 0 : k];
    __syncthreads();
    if (wv == 0 && unit) {
      float v = s_red[0][lane];
#pragma unroll
      for (int w = 1; w < kDaWaves; ++w) v += s_red[w][lane];
      const int row = radial ? k : nr + k;
      partial[(size_t(blockIdx.x) * (nr + H) + row) * F + lane] = v;
    }
  }
}

// ---- per source: dPs[s] = sum of dhid over the edges out of s, and the
// weights in the order of the edges sorted by source; one wave a node
__global__ __launch_bounds__(256) void k_att_dps(int N, int F, int H, const int32_t* __restrict__ offsets,
                                                 const int32_t* __restrict__ perm, const float* __restrict__ dhid,
                                                 const float* __restrict__ alpha_eid, float* __restrict__ dPs,
                                                 float* __restrict__ alpha_src) {
  const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (s >= N) return;
  const int e0 = offsets[s], e1 = offsets[s + 1];
  for (int i = e0 * H + lane; i < e1 * H; i += kWave)
    alpha_src[i] = alpha_eid[size_t(perm[i / H]) * H + i % H];
  float v = 0.f;
  if (lane < F) {
    for (int e = e0; e < e1; ++e) v += dhid[size_t(perm[e]) * F + lane];
    dPs[size_t(s) * F + lane] = v;
  }
}

// ---- grad_x of the degree-0 rows: += dPt[n] W1[0 .. C)^T + dPs[n] W1[C .. 2C)^T;
// a workgroup takes 16 nodes, a thread one channel
constexpr int kDxNodes = 16;
__global__ __launch_bounds__(256) void k_att_dx0(int N, int d, int C, int F, const float* __restrict__ W1,
                                                 const float* __restrict__ dPt, const float* __restrict__ dPs,
                                                 float* __restrict__ grad_x) {
  __shared__ float st[kDxNodes][kMaxF], ss[kDxNodes][kMaxF];
  const int n0 = blockIdx.x * kDxNodes, cnt = min(kDxNodes, N - n0);
  for (int i = threadIdx.x; i < cnt * F; i += 256) {
    st[i / F][i % F] = dPt[size_t(n0) * F + i];
    ss[i / F][i % F] = dPs[size_t(n0) * F + i];
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= C) return;
  float acc[kDxNodes];
#pragma unroll
  for (int k = 0; k < kDxNodes; ++k) acc[k] = 0.f;
  for (int j = 0; j < F; ++j) {
    const float wt = W1[size_t(c) * F + j], ws = W1[size_t(C + c) * F + j];
#pragma unroll
    for (int k = 0; k < kDxNodes; ++k) acc[k] = fmaf(ws, ss[k][j], fmaf(wt, st[k][j], acc[k]));
  }
#pragma unroll
  for (int k = 0; k < kDxNodes; ++k)
    if (k < cnt) grad_x[size_t(n0 + k) * d * C + c] += acc[k];
}

// ---- the node rows of grad W1, x[:, 0]^T [dPt, dPs], in 32x32x2 fp32 MFMA:
// one 32 x 32 tile a wave over a range of nodes, partial [gridDim.y][2 C][F]
__global__ __launch_bounds__(256) void k_att_dw1(int N, int d, int C, int F, const float* __restrict__ x,
                                                 const float* __restrict__ dPt, const float* __restrict__ dPs,
                                                 float* __restrict__ partial) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, l32 = lane & 31;
  const int ft_n = (F + 31) / 32, ct_n = C / kTile;
  const int t = blockIdx.x * 4 + wave;
  if (t >= 2 * ct_n * ft_n) return;
  const int ft = t % ft_n, ct = (t / ft_n) % ct_n, which = t / (ft_n * ct_n);
  const int c = ct * kTile + l32, f = ft * kTile + l32;
  const float* P = which == 0 ? dPt : dPs;
  const int n0 = int(int64_t(blockIdx.y) * N / gridDim.y), n1 = int(int64_t(blockIdx.y + 1) * N / gridDim.y);
  f32x16 acc = f32x16{};
  for (int n = n0; n < n1; n += 16) {
    float av[8], bv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int nn = n + 2 * k + h;
      av[k] = nn < n1 ? x[size_t(nn) * d * C + c] : 0.f;
      bv[k] = nn < n1 && f < F ? P[size_t(nn) * F + f] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) acc = mfma32(av[k], bv[k], acc);
  }
  if (f >= F) return;
#pragma unroll
  for (int v = 0; v < 16; ++v)
    partial[(size_t(blockIdx.y) * 2 * C + which * C + ct * kTile + acc_row(v, h)) * F + f] = acc[v];
}

template <int L>
hipError_t launch_dg_l(const AttBwdArgs& a, const DgArgs& g, hipStream_t s) {
  const int blocks = (g.n_range * g.RT + 3) / 4, ct = a.C / kTile;
  if (ct <= 2)
    k_att_dg<L, 2><<<dim3(blocks), dim3(256), 0, s>>>(g);
  else if (ct <= 4)
    k_att_dg<L, 4><<<dim3(blocks), dim3(256), 0, s>>>(g);
  else
    k_att_dg<L, 8><<<dim3(blocks), dim3(256), 0, s>>>(g);
  return hipGetLastError();
}
template <int L>
hipError_t launch_g_l(const AttBwdArgs& a, hipStream_t s) {
  k_att_g<L><<<dim3((a.E + kGEdges - 1) / kGEdges), dim3((a.R + 63) / 64 * 64), 0, s>>>(
      a.E, a.R, a.n_radial, a.sigma, a.perm, a.edge_vec, a.B, a.radial_w, a.g);
  return hipGetLastError();
}

}  // namespace

size_t att_bwd_ops_bytes(int d, int R) {
  const int RT = (R + kTile - 1) / kTile;
  return size_t(2) * pk_blocks(d) * RT * kWave * 16 + size_t(2) * RT * kTile * 4;
}
int att_bwd_da_blocks(int N) {
  const int b = (N + kDaWaves - 1) / kDaWaves, most = 4 * device_cus();
  return b < most ? b : most;
}
int att_bwd_dw1_parts(int N) {
  const int b = (N + 63) / 64;
  return b < 1 ? 1 : (b < 64 ? b : 64);
}

hipError_t launch_att_bwd_dg(const AttBwdArgs& a, hipStream_t s) {
  if (a.E == 0) return hipSuccess;
  const int ct = a.C / kTile;
  if (a.L < 1 || a.L > 4 || a.C % kTile || ct > 8 || a.H < 1 || a.H > kMaxH || ct % a.H || a.R < 1 || a.R > 256 ||
      a.n_radial > kMaxRadial)
    return hipErrorInvalidValue;
  const int d = a.d, RT = (a.R + kTile - 1) / kTile;
  u32x4* ops = static_cast<u32x4*>(a.ops);
  float* f_scale = reinterpret_cast<float*>(ops + size_t(2) * pk_blocks(d) * RT * kWave);
  k_att_factors<<<dim3((2 * RT * kWave + 255) / 256), dim3(256), 0, s>>>(d, a.R, RT, a.A, a.D, ops, f_scale);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  switch (a.L) {
    case 1: e = launch_g_l<1>(a, s); break;
    case 2: e = launch_g_l<2>(a, s); break;
    case 3: e = launch_g_l<3>(a, s); break;
    default: e = launch_g_l<4>(a, s); break;
  }
  if (e != hipSuccess) return e;
  DgArgs g{};
  g.E = a.E;
  g.C = a.C;
  g.R = a.R;
  g.RT = RT;
  g.H = a.H;
  // two waves a SIMD up to 128 channels, one above (registers)
  const int waves = device_cus() * (ct <= 4 ? 8 : 4), ranges = waves / RT;
  g.n_range = ranges < 1 ? 1 : (ranges < a.E ? ranges : a.E);
  g.perm = a.perm;
  g.src = a.src;
  g.dst = a.dst;
  g.xp = static_cast<const uint32_t*>(a.xp);
  g.gp = static_cast<const uint32_t*>(a.gp);
  g.x_scale = a.x_scale;
  g.g_scale = a.g_scale;
  g.ops = ops;
  g.f_scale = f_scale;
  g.g = a.g;
  g.alpha = a.alpha;
  g.dg = a.dg;
  g.dal = a.dal;
  switch (a.L) {
    case 1: return launch_dg_l<1>(a, g, s);
    case 2: return launch_dg_l<2>(a, g, s);
    case 3: return launch_dg_l<3>(a, g, s);
    default: return launch_dg_l<4>(a, g, s);
  }
}

hipError_t launch_att_bwd_mlp(const AttBwdArgs& a, hipStream_t s) {
  if (a.F < 1 || a.F > kMaxF || a.H < 1 || a.H > kMaxH || a.n_radial < 1 || a.n_radial > kMaxRadial || a.C > 256 ||
      a.C % kTile)
    return hipErrorInvalidValue;
  const int nb = att_bwd_da_blocks(a.N), rows = a.n_radial + a.H;
  k_att_da<<<dim3(nb), dim3(kDaWaves * kWave), 0, s>>>(
      a.N, a.E, a.C, a.F, a.H, a.n_radial, (a.R + kTile - 1) / kTile, a.sigma, a.offsets, a.perm, a.src, a.edge_vec,
      a.Pt, a.Ps, a.W1, a.w2, a.alpha, a.dal, a.dhid, a.dPt, a.grad_vec, a.part_da);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_att_dps<<<dim3((a.N + 3) / 4), dim3(256), 0, s>>>(a.N, a.F, a.H, a.off_src, a.perm_src, a.dhid, a.alpha_eid, a.dPs,
                                                      a.alpha_src);
  e = hipGetLastError();
  if (e != hipSuccess || (!a.grad_w1 && !a.grad_w2)) return e;
  // the sums of the workgroups' radial rows and grad w2 (as [H][F]), then both to their places
  e = launch_sum_parts(nb, rows * a.F, a.part_da, a.sum_da, s);
  if (e != hipSuccess) return e;
  if (a.grad_w1) {
    const int parts = att_bwd_dw1_parts(a.N), tiles = 2 * (a.C / kTile) * ((a.F + 31) / 32);
    k_att_dw1<<<dim3((tiles + 3) / 4, parts), dim3(256), 0, s>>>(a.N, a.d, a.C, a.F, a.x, a.dPt, a.dPs, a.part_w1);
    e = hipGetLastError();
    if (e == hipSuccess) e = launch_sum_parts(parts, 2 * a.C * a.F, a.part_w1, a.grad_w1, s);
    if (e != hipSuccess) return e;
  }
  return launch_att_bwd_place(a, s);
}

namespace {
// the radial rows of grad W1, and grad w2 [F, H] from its sums [H][F]
__global__ void k_att_place(int C, int F, int H, int nr, const float* __restrict__ sum, float* __restrict__ grad_w1,
                            float* __restrict__ grad_w2) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < nr * F && grad_w1) grad_w1[size_t(2 * C) * F + i] = sum[i];
  if (i < F * H && grad_w2) grad_w2[i] = sum[size_t(nr) * F + (i % H) * F + i / H];
}
}  // namespace

hipError_t launch_att_bwd_place(const AttBwdArgs& a, hipStream_t s) {
  const int n = a.F * (a.n_radial > a.H ? a.n_radial : a.H);
  k_att_place<<<dim3((n + 255) / 256), dim3(256), 0, s>>>(a.C, a.F, a.H, a.n_radial, a.sum_da, a.grad_w1, a.grad_w2);
  return hipGetLastError();
}

hipError_t launch_att_bwd_x0(const AttBwdArgs& a, float* grad_x, hipStream_t s) {
  k_att_dx0<<<dim3((a.N + kDxNodes - 1) / kDxNodes), dim3(256), 0, s>>>(a.N, a.d, a.C, a.F, a.W1, a.dPt, a.dPs, grad_x);
  return hipGetLastError();
}

}  // namespace tdn
