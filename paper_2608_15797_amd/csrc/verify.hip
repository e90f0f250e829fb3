// Drafted tokens checked against the target's distribution, and the next token
// drawn (speculative sampling: the tokens are distributed as if the target had
// sampled each of them).
//
// P_t and Q_t are what the sampler would draw from for the target's and the
// draft's logits at position t: the top_k largest logits, ties to the lower
// id, their softmax at the temperature, the shortest prefix that reaches
// top_p, renormalised. So both are lists of at most 64 tokens, and everything
// after the lists is found is small enough for float64: decisions fall as in
// exact arithmetic.
//
// Two launches: the lists of every split of every row, each with a threshold
// that passes over nearly all logits by one compare; then a workgroup per
// sequence merges the splits' lists, a wave per row, and one wave goes through
// the positions.
#include <hip/hip_runtime.h>

#include "entropy_common.h"
#include "kvr_device.h"
#include "kvr_internal.h"
#include "sampler_common.h"

namespace kvr {

namespace {

constexpr int kThreads = 256;
constexpr int kMergeWaves = 8;
constexpr int kListMax = 1024;  // splits * top_k bound of a row's merge

// Row r of the call: the S (T + 1) target rows, then the S T draft rows.
struct Row {
  const char *x;
  int V, top_k;
  bool live;
};
__device__ __forceinline__ Row row_of(const VerifyParams &p, int r, int esz) {
  const int nt = p.S * (p.T + 1);
  const bool draft = r >= nt;
  const int q = draft ? r - nt : r, per = draft ? p.T : p.T + 1;
  const int s = q / per, t = q % per;
  const int nd = p.n_draft ? min(max(p.n_draft[s], 0), p.T) : p.T;
  Row o;
  o.live = draft ? t < nd : t <= nd;
  o.x = static_cast<const char *>(draft ? p.draft : p.logits) + (size_t)q * (draft ? p.ldd : p.ld) * esz;
  o.V = draft ? p.Vd : p.V;
  o.top_k = draft ? p.top_kd : p.top_k;
  return o;
}

// The keys of a row's splits in the workspace: [row][split][kmax].
__device__ __forceinline__ uint64_t *list_at(const VerifyParams &p, int r, int split) {
  const int kmax = max(p.top_k, p.top_kd);
  return p.ws + ((size_t)r * p.splits + split) * kmax;
}

// One split of a row: its top_k keys, in any order, zeros after them.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_split(VerifyParams p) {
  constexpr int NW = kThreads / kWave;
  __shared__ uint64_t cand[NW * kCandCap];
  __shared__ int cand_n[NW];
  const int split = blockIdx.x % p.splits, r = blockIdx.x / p.splits;
  const Row row = row_of(p, r, sizeof(T));
  if (!row.live) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, K = row.top_k;
  const T *x = reinterpret_cast<const T *>(row.x);
  const int per = (row.V + p.splits - 1) / p.splits;
  const int e0 = min(split * per, row.V), e1 = min(e0 + per, row.V);
  Cands cs{cand + wave * kCandCap, 0, 1, kNegInf};
  for (int eb = e0; eb < e1; eb += kThreads) {
    float a[8] = {kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf};
    const bool has = eb + tid < e1;
    if (has) a[0] = load1(x + eb + tid);
    cand_offer(cs, K, lane, a, (uint32_t)(eb + tid), has ? 1 : 0);
  }
  if (cs.cnt > K) cand_reduce_any(cs, K, K, lane);
  if (lane == 0) cand_n[wave] = cs.cnt;
  __syncthreads();
  if (wave != 0) return;
  int off[NW + 1];
  off[0] = 0;
#pragma unroll
  for (int w = 0; w < NW; w++) off[w + 1] = off[w] + cand_n[w];
  uint64_t *keys = list_at(p, r, split);
  const int nk = gather_select<NW * kTopKMax / kWave, NW>(cand, off, K, lane, keys);
  for (int q = nk + lane; q < K; q += kWave) keys[q] = 0;
}

// A distribution as a list: lane i holds token i, by falling probability.
struct Dist {
  int id;      // -1: no token
  double p;
};

// The k best keys of the row's splits, sorted over the lanes, by one wave.
__device__ __forceinline__ uint64_t merge_keys(const VerifyParams &p, int r, int k, int lane, uint64_t *tmp) {
  constexpr int NPL = kListMax / kWave;
  const uint64_t *src = list_at(p, r, 0);
  const int kmax = max(p.top_k, p.top_kd);
  uint64_t v[NPL];
#pragma unroll
  for (int i = 0; i < NPL; i++) {
    const int e = lane + i * kWave, split = e / k;
    v[i] = split < p.splits ? src[(size_t)split * kmax + e % k] : 0;
  }
  const uint64_t thr = select_threshold<NPL>(v, k, k);
  wave_lds_sync();
  const int n = wave_store_ge<NPL>(tmp, v, thr, lane);
  wave_lds_sync();
  const uint64_t key = lane < n ? tmp[lane] : 0;
  int rank = 0;
  for (int j = 0; j < n; j++) rank += tmp[j] > key;
  wave_lds_sync();
  if (lane < n) tmp[rank] = key;
  wave_lds_sync();
  return lane < n ? tmp[lane] : 0;
}

__device__ __forceinline__ double lane_cumsum(double x, int lane) {
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const double o = __shfl_up(x, off, kWave);
    if (lane >= off) x += o;
  }
  return x;
}

// The sampler's distribution of sorted keys.
__device__ __forceinline__ Dist distribution(uint64_t key, double temp, double top_p, int lane) {
  const bool live = key != 0;
  const float x = live ? from_order_bits((uint32_t)(key >> 32)) : kNegInf;
  const float x0 = __shfl(x, 0, kWave);
  double w = live && x > kNegInf ? exp(((double)x - (double)x0) / temp) : 0.0;
  double cum = lane_cumsum(w, lane);
  const double all = __shfl(cum, kWave - 1, kWave);
  const uint64_t reach = __ballot(cum >= top_p * all);
  const int keep = reach ? __ffsll((long long)reach) : kWave;  // tokens of the nucleus
  if (lane >= keep) w = 0.0;
  const double mass = __shfl(cum, keep - 1, kWave);
  return Dist{live && lane < keep ? (int)~(uint32_t)(key & 0xffffffffu) : -1, w / mass};
}

__global__ __launch_bounds__(kMergeWaves * kWave) void verify_walk(VerifyParams p) {
  extern __shared__ char lds[];
  const int s = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int nd = p.n_draft ? min(max(p.n_draft[s], 0), p.T) : p.T;
  // Probabilities and ids of the target's rows, then of the draft's; scratch of the merges.
  const int rows = 2 * p.T + 1;
  double *prob = reinterpret_cast<double *>(lds);
  int *ids = reinterpret_cast<int *>(prob + (size_t)rows * kWave);
  uint64_t *tmp = reinterpret_cast<uint64_t *>(ids + (size_t)rows * kWave) + wave * kWave;
  const int live = nd + 1 + (p.draft ? nd : 0);
  for (int i = wave; i < live; i += kMergeWaves) {
    const bool draft = i > nd;
    const int t = draft ? i - nd - 1 : i;
    const int r = draft ? p.S * (p.T + 1) + s * p.T + t : s * (p.T + 1) + t;
    const uint64_t key = merge_keys(p, r, draft ? p.top_kd : p.top_k, lane, tmp);
    const Dist d = distribution(key, draft ? p.tempd : p.temp, draft ? p.top_pd : p.top_p, lane);
    const int at = (draft ? p.T + 1 + t : t) * kWave + lane;
    prob[at] = d.p;
    ids[at] = d.id;
  }
  __syncthreads();
  if (wave != 0) return;
  int32_t *out = p.tokens + (size_t)s * (p.T + 1);
  int acc = 0;
  double r = 0.0;
  for (; acc < nd; acc++) {
    const int tok = p.tok[(size_t)s * p.T + acc];
    const double P = prob[acc * kWave + lane];
    const int id = ids[acc * kWave + lane];
    const double Pd = p.draft ? prob[(p.T + 1 + acc) * kWave + lane] : (lane == 0 ? 1.0 : 0.0);
    const int jd = p.draft ? ids[(p.T + 1 + acc) * kWave + lane] : (lane == 0 ? tok : -1);
    // The two probabilities of the drafted token: at most one lane of each has it.
    const uint64_t ip = __ballot(id == tok && id >= 0), iq = __ballot(jd == tok && jd >= 0);
    const double px = ip ? __shfl(P, __ffsll((long long)ip) - 1, kWave) : 0.0;
    const double qx = iq ? __shfl(Pd, __ffsll((long long)iq) - 1, kWave) : 0.0;
    if ((double)p.u_accept[(size_t)s * p.T + acc] * qx < px) {
      if (lane == 0) out[acc] = tok;
      continue;
    }
    // What the target has beyond the draft.
    double q = 0.0;
    for (int j = 0; j < kWave; j++) {
      const int other = __shfl(jd, j, kWave);
      const double oq = __shfl(Pd, j, kWave);
      if (other == id && id >= 0) q = oq;
    }
    r = id >= 0 ? fmax(P - q, 0.0) : 0.0;
    break;
  }
  const double P = prob[acc * kWave + lane];
  const int id = ids[acc * kWave + lane];
  if (acc == nd || !__any(r > 0.0)) r = P;
  const double cum = lane_cumsum(r, lane);
  const double all = __shfl(cum, kWave - 1, kWave);
  const uint64_t over = __ballot(r > 0.0 && cum > (double)p.u_draw[s] * all);
  const uint64_t any = __ballot(r > 0.0);
  const int pick = over ? __ffsll((long long)over) - 1 : any ? 63 - __clzll((long long)any) : 0;
  const int next = __shfl(id, pick, kWave);
  for (int t = acc + lane; t <= p.T; t += kWave) out[t] = t == acc ? next : -1;
  if (lane == 0) {
    p.accepted[s] = acc;
    if (p.len_out) p.len_out[s] = p.len[s] - (nd - acc);
  }
}

int verify_splits(int S, int T, int V, int Vd, int top_k) {
  const int rows = S * (2 * T + 1), vmax = V > Vd ? V : Vd;
  int n = (1024 + rows - 1) / rows;
  const int most = kListMax / top_k, useful = (vmax + 8191) / 8192;
  n = n < useful ? n : useful;
  n = n < most ? n : most;
  return n < 1 ? 1 : n;
}

}  // namespace

size_t verify_workspace_bytes(int S, int T, int V, int Vd, int top_k) {
  return (size_t)S * (2 * T + 1) * verify_splits(S, T, V, Vd, top_k) * top_k * sizeof(uint64_t);
}

hipError_t launch_verify_draft(const VerifyParams &params, hipStream_t stream) {
  VerifyParams p = params;
  const int k = p.top_k > p.top_kd ? p.top_k : p.top_kd;
  p.splits = verify_splits(p.S, p.T, p.V, p.Vd, k);
  const int rows = p.S * (p.T + 1) + (p.draft ? p.S * p.T : 0);
  const dim3 grid((uint32_t)rows * p.splits);
  if (p.dtype == 0) hipLaunchKernelGGL(verify_split<float>, grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL(verify_split<bf16_t>, grid, dim3(kThreads), 0, stream, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t lds = (size_t)(2 * p.T + 1) * kWave * (sizeof(double) + sizeof(int)) +
                     (size_t)kMergeWaves * kWave * sizeof(uint64_t);
  hipLaunchKernelGGL(verify_walk, dim3(p.S), dim3(kMergeWaves * kWave), lds, stream, p);
  return hipGetLastError();
}

}  // namespace kvr
