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

#include <type_traits>

#include "entropy_common.h"
#include "kvr_device.h"
#include "kvr_internal.h"
#include "sampler_common.h"

namespace kvr {

namespace {

constexpr int kThreads = 256;
constexpr int kMergeWaves = 16;
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

// The top_k best keys of a workgroup's wave buffers, sorted, zeros after them.
template <int NW>
__device__ __forceinline__ void write_best(Cands &cs, uint64_t *cand, int *cand_n, int K, int lane, int wave,
                                           uint64_t *keys) {
  __shared__ uint64_t best[kTopKMax];
  if (cs.cnt > K) cand_reduce_any(cs, K, K, lane);
  if (lane == 0) cand_n[wave] = cs.cnt;
  __syncthreads();
  if (wave != 0) return;
  int off[NW + 1];
  off[0] = 0;
#pragma unroll
  for (int w = 0; w < NW; w++) off[w + 1] = off[w] + cand_n[w];
  const int n = gather_select<NW * kTopKMax / kWave, NW>(cand, off, K, lane, best);
  wave_lds_sync();
  const uint64_t key = lane < n ? best[lane] : 0;
  int rank = 0;
  for (int j = 0; j < n; j++) rank += best[j] > key;
  if (lane < n) keys[rank] = key;
  else if (lane < K) keys[lane] = 0;
}

constexpr int kU = 10;                        // vectors of eight logits per thread
constexpr int kRoundVecs = kThreads * kU;

// One split of a row, all of its logits in registers at once: its top_k keys,
// sorted, zeros after them. The top_k-th largest of the 256 lanes' maxima (16
// leading bits of it) bounds the split's top_k-th best from below, so about
// top_k logits are candidates and most vectors are passed over by one compare;
// they are ranked by counting. Where they outnumber the threads (many equal
// logits) or too few lanes hold a logit for a bound, the waves' buffers take
// them, from the same registers.
template <typename T>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 5 : 4))) void verify_split(VerifyParams p) {
  constexpr int U = kU, NT = kThreads, NW = NT / kWave;
  __shared__ uint32_t lane_max[NT];
  __shared__ __align__(16) uint64_t cand[NW * kCandCap];
  __shared__ int count, cand_n[NW];
  static_assert(NW * kCandCap >= NT && NT % 8 == 0, "a candidate per thread, ranked in eights");
  const int split = blockIdx.x % p.splits, r = blockIdx.x / p.splits;
  const Row row = row_of(p, r, sizeof(T));
  if (!row.live) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, K = row.top_k;
  const T *x = reinterpret_cast<const T *>(row.x);
  // Vectors from the row's first 16-byte boundary, element `skip`; the logits
  // before it and the last few one per thread of the last split's first wave.
  const int skip = min((int)((0 - reinterpret_cast<uintptr_t>(x)) % 16 / sizeof(T)), row.V);
  const int nvec = (row.V - skip) / 8, per = (nvec + p.splits - 1) / p.splits;
  const int v0 = min(split * per, nvec), v1 = min(v0 + per, nvec);
  const rsrc_t rr = row_rsrc(x + skip, (uint32_t)v1 * 8u * (uint32_t)sizeof(T));
  Vec8<T> w[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    w[u].load(rr, v0 + tid + u * NT);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (tid == 0) count = 0;
  cand[tid] = 0;
  float lm[U], mx = kNegInf;
#pragma unroll
  for (int u = 0; u < U; u++) {
    float a[8];
    w[u].get(a);
    lm[u] = kNegInf;
    if (v0 + tid + u * NT < v1) {
#pragma unroll
      for (int e = 0; e < 8; e++) lm[u] = fmaxf(lm[u], a[e]);  // a NaN is passed over
    }
    mx = fmaxf(mx, lm[u]);
  }
  const int et = tid < skip ? tid : nvec * 8 + tid;
  const bool has_tail = split == p.splits - 1 && et < row.V && tid < kWave;
  const float tail = has_tail ? load1(x + et) : kNegInf;
  mx = fmaxf(mx, tail);
  lane_max[tid] = order_bits(mx);
  __syncthreads();

  const float vmin = group_bound<NW>(lane_max, lane, K);  // nothing below it is among the split's best
  bool over = vmin == kNegInf;
  if (over) count = NT + 1;
  auto offer = [&](float v, uint32_t id) {
    const int at = atomicAdd(&count, 1);
    if (at < NT) cand[at] = cand_key(v, id);
    over = at >= NT;
  };
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int v = v0 + tid + u * NT;
    if (v < v1 && !over && lm[u] >= vmin) {
      float a[8];
      w[u].get(a);
#pragma unroll
      for (int e = 0; e < 8; e++)
        if (!over && a[e] >= vmin) offer(a[e], (uint32_t)(skip + v * 8 + e));
    }
  }
  if (has_tail && !over && tail >= vmin) offer(tail, (uint32_t)et);
  __syncthreads();

  uint64_t *keys = list_at(p, r, split);
  const int n = count;
  if (n <= NT) {
    // Counting gives the same order whatever the order of the atomics.
    const uint64_t key = tid < n ? cand[tid] : 0;
    int rank = 0;
    for (int j = 0; j < n; j += 8)
#pragma unroll
      for (int q = 0; q < 8; q++) rank += cand[j + q] > key;  // zeros past the last
    if (tid < n) {
      if (rank < K) keys[rank] = key;
    } else if (tid < K) {
      keys[tid] = 0;
    }
    return;
  }
  Cands cs{cand + wave * kCandCap, 0, 1, kNegInf};
  __syncthreads();  // every thread is past its read of the count and the candidates
  cand_seed(cs, mx, K);
#pragma unroll 1
  for (int u = 0; u < U; u++) {
    float a[8];
    Vec8<T> wu = w[0];
#pragma unroll
    for (int q = 1; q < U; q++)
      if (q == u) wu = w[q];
    wu.get(a);
    const int v = v0 + tid + u * NT;
    cand_offer(cs, K, lane, a, (uint32_t)(skip + v * 8), v < v1 ? 8 : 0);
  }
  float a[8] = {tail, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf};
  if (wave == 0) cand_offer(cs, K, lane, a, (uint32_t)et, has_tail ? 1 : 0);
  write_best<NW>(cs, cand, cand_n, K, lane, wave, keys);
}

// One split of a row of more logits than that, streamed.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_stream(VerifyParams p) {
  constexpr int NW = kThreads / kWave;
  __shared__ uint64_t cand[NW * kCandCap];
  __shared__ int cand_n[NW];
  const int split = blockIdx.x % p.splits, r = blockIdx.x / p.splits;
  const Row row = row_of(p, r, sizeof(T));
  if (!row.live) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, K = row.top_k;
  const T *x = reinterpret_cast<const T *>(row.x);
  const int per = (row.V + p.splits - 1) / p.splits;
  const int e0 = min((long)split * per, (long)row.V), e1 = min((long)e0 + per, (long)row.V);
  Cands cs{cand + wave * kCandCap, 0, 1, kNegInf};
  for (int eb = e0; eb < e1; eb += kThreads) {
    float a[8] = {kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf, kNegInf};
    const bool has = eb + tid < e1;
    if (has) a[0] = load1(x + eb + tid);
    cand_offer(cs, K, lane, a, (uint32_t)(eb + tid), has ? 1 : 0);
  }
  write_best<NW>(cs, cand, cand_n, K, lane, wave, list_at(p, r, split));
}

// A distribution as a list: lane i holds token i, by falling probability.
struct Dist {
  int id;      // -1: no token
  double p;
};

// The word of lane ^ M, without LDS (a workgroup's waves merge at once).
template <int M>
__device__ __forceinline__ uint32_t exchange(uint32_t x) {
  auto dpp = [](uint32_t v, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  if constexpr (M == 1) return dpp(x, std::integral_constant<int, 0xb1>());
  if constexpr (M == 2) return dpp(x, std::integral_constant<int, 0x4e>());
  // Lane ^ 3 within four lanes, lane ^ 7 within eight.
  if constexpr (M == 4) return dpp(dpp(x, std::integral_constant<int, 0x1b>()), std::integral_constant<int, 0x141>());
  if constexpr (M == 8) return dpp(x, std::integral_constant<int, 0x128>());  // by 8 around 16
#if defined(__HIP_DEVICE_COMPILE__)
  // The rows (halves) of x and of its copy change places: one holds the even ones twice, one the odd.
  const bool odd = threadIdx.x & M;
  if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return odd ? r[0] : r[1];
  }
  if constexpr (M == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return odd ? r[0] : r[1];
  }
#endif
  return x;
}

// Keys M lanes apart in order: the larger first, with `up` last.
template <int M>
__device__ __forceinline__ uint64_t order(uint64_t x, bool up) {
  const uint64_t o = exchange<M>((uint32_t)x) | ((uint64_t)exchange<M>((uint32_t)(x >> 32)) << 32);
  const bool less = ((threadIdx.x & M) != 0) != up;  // this lane takes the smaller one
  return (x < o) == less ? x : o;
}

// Runs of SIZE lanes that fall and then rise (or rise and then fall), sorted:
// rising where `up` says so.
template <int SIZE>
__device__ __forceinline__ uint64_t sort_runs(uint64_t x, bool up) {
  if constexpr (SIZE >= 64) x = order<32>(x, up);
  if constexpr (SIZE >= 32) x = order<16>(x, up);
  if constexpr (SIZE >= 16) x = order<8>(x, up);
  if constexpr (SIZE >= 8) x = order<4>(x, up);
  if constexpr (SIZE >= 4) x = order<2>(x, up);
  return order<1>(x, up);
}

// The k best keys of the row's splits, sorted over the lanes, by one wave. A
// register holds as many of the splits' sorted lists as fit its lanes, every
// other one rising, and is sorted from there; NB registers are then joined in
// pairs, one falling and one rising: the larger of each lane's two keys are the
// best of both.
template <int NB>
__device__ __forceinline__ uint64_t merge_keys(const VerifyParams &p, int r, int k, int lane) {
  const uint64_t *src = list_at(p, r, 0);
  const int kmax = max(p.top_k, p.top_kd);
  const int log_kp = k > 1 ? 32 - __clz(k - 1) : 0, kp = 1 << log_kp;  // lanes of a list
  uint64_t best = 0;
  for (int s0 = 0; s0 < p.splits; s0 += NB * kWave >> log_kp) {
    uint64_t v[NB];
#pragma unroll
    for (int i = 0; i < NB; i++) {
      const int e = i * kWave + lane, split = s0 + (e >> log_kp);
      const int at = (e >> log_kp) & 1 ? kp - 1 - (e & (kp - 1)) : e & (kp - 1);
      v[i] = split < p.splits && at < k ? src[(size_t)split * kmax + at] : 0;
    }
#define KVR_SORT(SIZE)                                                                                    \
    if (kp < SIZE)                                                                                        \
      _Pragma("unroll") for (int i = 0; i < NB; i++) v[i] = sort_runs<SIZE>(v[i], (i * kWave + lane) & SIZE);
    KVR_SORT(2) KVR_SORT(4) KVR_SORT(8) KVR_SORT(16) KVR_SORT(32) KVR_SORT(64)
#undef KVR_SORT
#pragma unroll
    for (int n = NB / 2; n >= 1; n /= 2)
#pragma unroll
      for (int i = 0; i < n; i++)
        v[i] = sort_runs<kWave>(max(v[2 * i], v[2 * i + 1]), n > 1 ? i & 1 : s0 > 0);
    best = s0 == 0 ? v[0] : sort_runs<kWave>(max(best, v[0]), false);
  }
  return lane < k ? best : 0;
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

// The lists of a sequence's rows, a wave per row; then one wave goes through the
// positions. NB: registers of lists merged at once.
template <int NB>
__global__ __launch_bounds__(kMergeWaves * kWave) void verify_walk(VerifyParams p) {
  extern __shared__ char lds[];
  __shared__ int stands[kWave];  // T is at most 32
  const int s = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int nd = p.n_draft ? min(max(p.n_draft[s], 0), p.T) : p.T;
  // Probabilities and ids of the target's rows, then of the draft's.
  const int rows = 2 * p.T + 1;
  double *prob = reinterpret_cast<double *>(lds);
  int *ids = reinterpret_cast<int *>(prob + (size_t)rows * kWave);
  const int live = nd + 1 + (p.draft ? nd : 0);
  for (int i = wave; i < live; i += kMergeWaves) {
    const bool draft = i > nd;
    const int t = draft ? i - nd - 1 : i;
    const int r = draft ? p.S * (p.T + 1) + s * p.T + t : s * (p.T + 1) + t;
    const uint64_t key = merge_keys<NB>(p, r, draft ? p.top_kd : p.top_k, lane);
    const Dist d = distribution(key, draft ? p.tempd : p.temp, draft ? p.top_pd : p.top_p, lane);
    const int at = (draft ? p.T + 1 + t : t) * kWave + lane;
    prob[at] = d.p;
    ids[at] = d.id;
  }
  __syncthreads();
  // Which of the drafted tokens would stand by themselves, a wave per position.
  for (int t = wave; t < nd; t += kMergeWaves) {
    const int tok = p.tok[(size_t)s * p.T + t];
    const float ua = p.u_accept[(size_t)s * p.T + t];
    const uint64_t ip = __ballot(ids[t * kWave + lane] == tok && tok >= 0);
    const double px = ip ? prob[t * kWave + __ffsll((long long)ip) - 1] : 0.0;
    double qx = 1.0;
    if (p.draft) {
      const uint64_t iq = __ballot(ids[(p.T + 1 + t) * kWave + lane] == tok && tok >= 0);
      qx = iq ? prob[(p.T + 1 + t) * kWave + __ffsll((long long)iq) - 1] : 0.0;
    }
    if (lane == 0) stands[t] = (double)ua * qx < px;
  }
  __syncthreads();
  if (wave != 0) return;
  int32_t *out = p.tokens + (size_t)s * (p.T + 1);
  const uint64_t fell = __ballot(lane < nd && !stands[lane]);
  const int acc = fell ? __ffsll((long long)fell) - 1 : nd;
  double r = 0.0;
  const double P = prob[acc * kWave + lane];
  const int id = ids[acc * kWave + lane];
  if (acc < nd) {
    // What the target has beyond the draft.
    double q = 0.0;
    if (p.draft) {
      const int at = (p.T + 1 + acc) * kWave, n = __popcll(__ballot(ids[at + lane] >= 0));  // the tokens come first
      for (int j = 0; j < n; j++)
        if (ids[at + j] == id) q = prob[at + j];
    } else if (id == p.tok[(size_t)s * p.T + acc]) {
      q = 1.0;
    }
    r = id >= 0 ? fmax(P - q, 0.0) : 0.0;
  }
  if (acc == nd || !__any(r > 0.0)) r = P;
  const double cum = lane_cumsum(r, lane);
  const double all = __shfl(cum, kWave - 1, kWave);
  const uint64_t over = __ballot(r > 0.0 && cum > (double)p.u_draw[s] * all);
  const uint64_t any = __ballot(r > 0.0);
  const int pick = over ? __ffsll((long long)over) - 1 : any ? 63 - __clzll((long long)any) : 0;
  const int next = __shfl(id, pick, kWave);
  for (int t = lane; t <= p.T; t += kWave) out[t] = t < acc ? p.tok[(size_t)s * p.T + t] : t == acc ? next : -1;
  if (lane == 0) {
    p.accepted[s] = acc;
    if (p.len_out) p.len_out[s] = p.len[s] - (nd - acc);
  }
}

// Lanes of a merge that a split's list takes.
int list_lanes(int top_k) {
  int lanes = 1;
  while (lanes < top_k) lanes *= 2;
  return lanes;
}

// Splits of a row: enough that a workgroup holds one at once, where the merge
// takes that many lists; with few rows more of them, up to 1024 workgroups and
// four registers of lists (9 rows of 152k logits, top 20: 16.3 us with 8 lists,
// 17.8 with 12, 24 with 25).
int verify_splits(int S, int T, int V, int Vd, int top_k) {
  const long rows = (long)S * (2 * T + 1), nvec = (V > Vd ? V : Vd) / 8;
  long n = (1024 + rows - 1) / rows;
  const long useful = (nvec + kThreads - 1) / kThreads, round = (nvec + kRoundVecs - 1) / kRoundVecs;
  const long lists = 4 * kWave / list_lanes(top_k);
  n = n < lists ? n : lists;
  n = n < useful ? n : useful;
  n = n > round ? n : round;
  n = n < kListMax / top_k ? n : kListMax / top_k;
  return n < 1 ? 1 : (int)n;
}

template <typename T>
void launch_rows(const VerifyParams &p, dim3 grid, hipStream_t stream) {
  if ((p.V / 8 + p.splits - 1) / p.splits <= kRoundVecs)
    hipLaunchKernelGGL(verify_split<T>, grid, dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL(verify_stream<T>, grid, dim3(kThreads), 0, stream, p);
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
  if (p.dtype == 0) launch_rows<float>(p, grid, stream);
  else launch_rows<bf16_t>(p, grid, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t lds = (size_t)(2 * p.T + 1) * kWave * (sizeof(double) + sizeof(int));
  const dim3 seqs(p.S), threads(kMergeWaves * kWave);
  const int regs = (p.splits * list_lanes(k) + kWave - 1) / kWave;
  if (regs <= 2) hipLaunchKernelGGL(verify_walk<2>, seqs, threads, lds, stream, p);
  else if (regs <= 4) hipLaunchKernelGGL(verify_walk<4>, seqs, threads, lds, stream, p);
  else hipLaunchKernelGGL(verify_walk<8>, seqs, threads, lds, stream, p);
  return hipGetLastError();
}

}  // namespace kvr
