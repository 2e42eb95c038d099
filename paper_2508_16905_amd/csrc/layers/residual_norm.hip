// r' = r + s g * P(b), y = N(r') and its gradients: one pass over the rows, a row in the registers of a team of lanes.
// Bound by memory: forward reads r and b and writes r' and y, backward reads dr', dy, r' and b and writes dr and db.  All
// sums are fp32; the statistics of the backward pass are computed again from the rows that it reads anyway.
#include "layer_util.h"
#include "layers.h"

namespace triaccel {
namespace layers {

namespace {

// Sums of N values over the T lanes of a team, in all its lanes.  T = 64: one wavefront; else the whole workgroup, through
// LDS; `turn` alternates between two places, so that one barrier per sum is enough.
template <int N>
__device__ __forceinline__ void wave_sum(float (&v)[N]) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], s, 64);
  }
}
template <int T, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* lds, int& turn) {
  wave_sum(v);
  if constexpr (T > 64) {
    constexpr int kWaves = T / 64;
    float* place = lds + turn * (4 * kWaves);
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) place[(threadIdx.x >> 6) * 4 + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s += place[w * 4 + i];
      v[i] = s;
    }
  }
}

// Mean (0 for RMS) and 1 / sqrt(variance + eps) of a row whose lanes hold V groups of eight, zeros past the end.
template <int T, int V>
__device__ __forceinline__ void statistics(int kind, const float (&x)[V][8], const bool (&in)[V], const int64_t (&left)[V], float cols, float eps,
                                           float* lds, int& turn, float& mean, float& rstd) {
  mean = 0.0f;
  if (kind == 2) {
    float s[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += x[v][i];
    team_sum<T>(s, lds, turn);
    mean = s[0] / cols;
  }
  float q[1] = {0.0f};
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = in[v] && i < left[v] ? x[v][i] - mean : 0.0f;
      q[0] = fmaf(d, d, q[0]);
    }
  team_sum<T>(q, lds, turn);
  rstd = 1.0f / sqrtf(q[0] / cols + eps);
}

__device__ __forceinline__ void vector8(const void* p, int dtype, int64_t col, int64_t left, float otherwise, float (&out)[8]) {
  if (p) {
    load8_of(dtype, p, col, left, out);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = otherwise;
  }
}

template <int DT, int T, int V>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_residual_norm(NormArgs a) {
  constexpr int kThreads = T < 256 ? 256 : T, kTeams = kThreads / T;
  __shared__ float lds[2 * 4 * (kThreads / 64)];
  const int lane = threadIdx.x % T;
  const int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / T;
  if (kTeams > 1 && row >= a.rows) return;  // a wavefront of its own: nobody waits for it
  int turn = 0;
  const float cols = (float)a.cols;
  int64_t col[V], left[V];
  bool in[V];
  float x[V][8], r[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    col[v] = ((int64_t)v * T + lane) * 8;
    left[v] = a.cols - col[v];
    in[v] = left[v] > 0;
    if (in[v]) {
      load8<DT>(a.r, row * a.ldr + col[v], left[v], r[v]);
      if (a.b) load8<DT>(a.b, row * a.ldb + col[v], left[v], x[v]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[v][i] = x[v][i] = 0.0f;
    }
  }
  if (a.b) {
    float mean = 0.0f, rstd = 1.0f;
    if (a.post.kind) statistics<T, V>(a.post.kind, x, in, left, cols, a.post.eps, lds, turn, mean, rstd);
    const int64_t gate_row = a.rows_per_gate ? row / a.rows_per_gate * a.ldgate : 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in[v]) continue;
      float w[8], c[8], g[8];
      if (a.post.kind) {
        vector8(a.post.weight, a.post.dtype, col[v], left[v], 1.0f, w);
        vector8(a.post.bias, a.post.dtype, col[v], left[v], 0.0f, c);
      }
      vector8(a.gate, a.gate_dtype, gate_row + col[v], left[v], 1.0f, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float p = x[v][i];
        if (a.post.kind) p = fmaf((p - mean) * rstd, w[i], c[i]);
        if (i < left[v]) r[v][i] = fmaf(a.scale * g[i], p, r[v][i]);
      }
      store8<DT>(a.ro, row * a.ldro + col[v], left[v], r[v]);
    }
  }
  if (!a.norm.kind) return;
  float mean, rstd;
  statistics<T, V>(a.norm.kind, r, in, left, cols, a.norm.eps, lds, turn, mean, rstd);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!in[v]) continue;
    float w[8], c[8], y[8];
    vector8(a.norm.weight, a.norm.dtype, col[v], left[v], 1.0f, w);
    vector8(a.norm.bias, a.norm.dtype, col[v], left[v], 0.0f, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fmaf((r[v][i] - mean) * rstd, w[i], c[i]);
    store8<DT>(a.y, row * a.ldy + col[v], left[v], y);
  }
}

// A team has a run of rows and keeps its columns' sums for the vectors' gradients in registers; a second kernel adds up the
// teams.  A gate with a row for each `rows_per_gate` rows is written where the team has all of these, and left in one of two
// places of the team (the group it begins in, another) where it has a part.
template <int DT, int T, int V>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_residual_norm_grad(NormGradArgs a) {
  constexpr int kThreads = T < 256 ? 256 : T, kTeams = kThreads / T;
  __shared__ float lds[2 * 4 * (kThreads / 64)];
  const int lane = threadIdx.x % T;
  const int64_t team = (int64_t)blockIdx.x * kTeams + threadIdx.x / T;
  if (kTeams > 1 && team >= a.teams) return;
  const int64_t r0 = team * a.rows_per_team, r1 = r0 + a.rows_per_team < a.rows ? r0 + a.rows_per_team : a.rows;
  int turn = 0;
  const float cols = (float)a.cols, inv = 1.0f / cols;
  const bool post = a.b && a.post.kind;
  int64_t col[V], left[V];
  bool in[V];
  float nw[V][8], nb[V][8], pw[V][8], pb[V][8], gs[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    col[v] = ((int64_t)v * T + lane) * 8;
    left[v] = a.cols - col[v];
    in[v] = left[v] > 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) nw[v][i] = nb[v][i] = pw[v][i] = pb[v][i] = gs[v][i] = 0.0f;
  }
  int64_t group = a.rows_per_gate ? r0 / a.rows_per_gate : 0;
  const int64_t first_group = group;
  const auto flush_gate = [&](int64_t g) {
    const int64_t g0 = g * a.rows_per_gate, g1 = g0 + a.rows_per_gate < a.rows ? g0 + a.rows_per_gate : a.rows;
    const bool whole = g0 >= r0 && g1 <= r1;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (in[v]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (i < left[v]) {
            if (whole) store1_of(a.vec_dtype, a.dgate, g * a.cols + col[v] + i, gs[v][i]);
            else as_global<float>(a.gate_edges)[(team * 2 + (g == first_group ? 0 : 1)) * a.cols + col[v] + i] = gs[v][i];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) gs[v][i] = 0.0f;
    }
  };
  for (int64_t row = r0; row < r1; ++row) {
    if (a.rows_per_gate && a.dgate) {
      const int64_t g = row / a.rows_per_gate;
      if (g != group) {
        flush_gate(group);
        group = g;
      }
    }
    float d[V][8], r[V][8], dy[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) d[v][i] = r[v][i] = dy[v][i] = 0.0f;
      if (in[v]) {
        if (a.dro) load8<DT>(a.dro, row * a.lddro + col[v], left[v], d[v]);
        if (a.norm.kind && a.dy) {
          load8<DT>(a.dy, row * a.lddy + col[v], left[v], dy[v]);
          load8<DT>(a.r, row * a.ldr + col[v], left[v], r[v]);
        }
      }
    }
    if (a.norm.kind && a.dy) {
      float mean, rstd;
      statistics<T, V>(a.norm.kind, r, in, left, cols, a.norm.eps, lds, turn, mean, rstd);
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8];
        if (in[v]) vector8(a.norm.weight, a.norm.dtype, col[v], left[v], 1.0f, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (!in[v] || i >= left[v]) continue;
          r[v][i] = (r[v][i] - mean) * rstd;
          nw[v][i] = fmaf(dy[v][i], r[v][i], nw[v][i]);
          nb[v][i] += dy[v][i];
          dy[v][i] *= w[i];
          s[0] = fmaf(dy[v][i], r[v][i], s[0]);
          s[1] += dy[v][i];
        }
      }
      team_sum<T>(s, lds, turn);
      const float along = s[0] * inv, centre = a.norm.kind == 2 ? s[1] * inv : 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (in[v] && i < left[v]) d[v][i] = fmaf(rstd, dy[v][i] - centre - r[v][i] * along, d[v][i]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (in[v] && a.dr) store8<DT>(a.dr, row * a.lddr + col[v], left[v], d[v]);
    if (!a.b) continue;
    // the block's side: t = P(b), dP = s g d
    float b[V][8], g[V][8];
    const int64_t gate_row = a.rows_per_gate ? row / a.rows_per_gate * a.ldgate : 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int i = 0; i < 8; ++i) b[v][i] = g[v][i] = 0.0f;
      if (in[v]) {
        if (a.b) load8<DT>(a.b, row * a.ldb + col[v], left[v], b[v]);
        vector8(a.gate, a.gate_dtype, gate_row + col[v], left[v], 1.0f, g[v]);
      }
    }
    float rstd = 1.0f, along = 0.0f, centre = 0.0f;
    if (post) {
      float mean;
      statistics<T, V>(a.post.kind, b, in, left, cols, a.post.eps, lds, turn, mean, rstd);
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8], c[8];
        if (in[v]) {
          vector8(a.post.weight, a.post.dtype, col[v], left[v], 1.0f, w);
          vector8(a.post.bias, a.post.dtype, col[v], left[v], 0.0f, c);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (!in[v] || i >= left[v]) continue;
          b[v][i] = (b[v][i] - mean) * rstd;
          const float t = fmaf(b[v][i], w[i], c[i]), dp = a.scale * g[v][i] * d[v][i];
          gs[v][i] = fmaf(a.scale * d[v][i], t, gs[v][i]);
          pw[v][i] = fmaf(dp, b[v][i], pw[v][i]);
          pb[v][i] += dp;
          d[v][i] = dp * w[i];
          s[0] = fmaf(d[v][i], b[v][i], s[0]);
          s[1] += d[v][i];
        }
      }
      team_sum<T>(s, lds, turn);
      along = s[0] * inv;
      centre = a.post.kind == 2 ? s[1] * inv : 0.0f;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          gs[v][i] = fmaf(a.scale * d[v][i], b[v][i], gs[v][i]);
          d[v][i] = a.scale * g[v][i] * d[v][i];
        }
    }
    if (a.db) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (post) {
#pragma unroll
          for (int i = 0; i < 8; ++i) d[v][i] = rstd * (d[v][i] - centre - b[v][i] * along);
        }
        if (in[v]) store8<DT>(a.db, row * a.lddb + col[v], left[v], d[v]);
      }
    }
  }
  if (a.rows_per_gate && a.dgate && r0 < r1) flush_gate(group);
  if (!a.sums) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!in[v]) continue;
    const int64_t at = team * kNormVectors * a.cols + col[v];
    if (a.dnw) store8<kFP32>(a.sums, at, left[v], nw[v]);
    if (a.dnb) store8<kFP32>(a.sums, at + a.cols, left[v], nb[v]);
    if (a.dpw) store8<kFP32>(a.sums, at + 2 * a.cols, left[v], pw[v]);
    if (a.dpb) store8<kFP32>(a.sums, at + 3 * a.cols, left[v], pb[v]);
    if (a.dgate && !a.rows_per_gate) store8<kFP32>(a.sums, at + 4 * a.cols, left[v], gs[v]);
  }
}

// The gates' gradients of groups of rows that more than one team had a part of, teams in order.
__global__ __launch_bounds__(256) void k_gate_groups(NormGradArgs a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t groups = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate;
  for (int64_t g = blockIdx.y; g < groups; g += gridDim.y) {
    const int64_t g0 = g * a.rows_per_gate, g1 = g0 + a.rows_per_gate < a.rows ? g0 + a.rows_per_gate : a.rows;
    const int64_t t0 = g0 / a.rows_per_team, t1 = (g1 - 1) / a.rows_per_team;
    if (t0 == t1) continue;  // written by its team
    float s = 0.0f;
    for (int64_t t = t0; t <= t1; ++t)
      s += as_global<float>(a.gate_edges)[(t * 2 + (t * a.rows_per_team / a.rows_per_gate == g ? 0 : 1)) * a.cols + c];
    store1_of(a.vec_dtype, a.dgate, g * a.cols + c, s);
  }
}

template <int DT>
hipError_t forward(const NormArgs& a, hipStream_t stream) {
  const uint32_t rows = (uint32_t)a.rows, quarter = (uint32_t)ceil_div(a.rows, 4);
  if (a.cols <= 512) k_residual_norm<DT, 64, 1><<<quarter, 256, 0, stream>>>(a);
  else if (a.cols <= 1024) k_residual_norm<DT, 64, 2><<<quarter, 256, 0, stream>>>(a);
  else if (a.cols <= 2048) k_residual_norm<DT, 256, 1><<<rows, 256, 0, stream>>>(a);
  else if (a.cols <= 4096) k_residual_norm<DT, 256, 2><<<rows, 256, 0, stream>>>(a);
  else if (a.cols <= 8192) k_residual_norm<DT, 512, 2><<<rows, 512, 0, stream>>>(a);
  else k_residual_norm<DT, 1024, 2><<<rows, 1024, 0, stream>>>(a);
  return hipGetLastError();
}
template <int DT>
hipError_t backward(const NormGradArgs& a, hipStream_t stream) {
  const uint32_t teams = (uint32_t)a.teams, quarter = (uint32_t)ceil_div(a.teams, 4);
  if (a.cols <= 512) k_residual_norm_grad<DT, 64, 1><<<quarter, 256, 0, stream>>>(a);
  else if (a.cols <= 1024) k_residual_norm_grad<DT, 64, 2><<<quarter, 256, 0, stream>>>(a);
  else if (a.cols <= 2048) k_residual_norm_grad<DT, 256, 1><<<teams, 256, 0, stream>>>(a);
  else if (a.cols <= 4096) k_residual_norm_grad<DT, 256, 2><<<teams, 256, 0, stream>>>(a);
  else if (a.cols <= 8192) k_residual_norm_grad<DT, 512, 2><<<teams, 512, 0, stream>>>(a);
  else k_residual_norm_grad<DT, 1024, 2><<<teams, 1024, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_residual_norm(int dtype, const NormArgs& a, hipStream_t stream) {
  return dtype == kFP16 ? forward<kFP16>(a, stream) : dtype == kBF16 ? forward<kBF16>(a, stream) : forward<kFP32>(a, stream);
}

void norm_grad_teams(int64_t rows, int64_t cols, int32_t& teams, int64_t& rows_per_team) {
  const int64_t most = cols <= 1024 ? 2048 : 512;
  rows_per_team = ceil_div(rows, most);
  if (rows_per_team < 1) rows_per_team = 1;
  teams = (int32_t)ceil_div(rows, rows_per_team);
}

hipError_t launch_residual_norm_grad(int dtype, const NormGradArgs& a, hipStream_t stream) {
  const hipError_t e = dtype == kFP16 ? backward<kFP16>(a, stream) : dtype == kBF16 ? backward<kBF16>(a, stream) : backward<kFP32>(a, stream);
  if (e != hipSuccess) return e;
  const bool grouped = a.dgate && a.rows_per_gate;
  if (grouped) {
    const int64_t groups = ceil_div(a.rows, a.rows_per_gate);
    k_gate_groups<<<dim3((uint32_t)ceil_div(a.cols, 256), (uint32_t)(groups < 4096 ? groups : 4096)), 256, 0, stream>>>(a);
  }
  if (a.dnw || a.dnb || a.dpw || a.dpb || (a.dgate && !grouped)) {
    ColumnSums s{a.sums, a.cols, kNormVectors * a.cols, a.teams, kNormVectors, a.vec_dtype, {a.dnw, a.dnb, a.dpw, a.dpb, grouped ? nullptr : a.dgate}};
    return launch_column_sums(s, stream);
  }
  return hipGetLastError();
}

}  // namespace layers
}  // namespace triaccel
