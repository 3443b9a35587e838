// Operators over the tokens of long videos: rotary positions, block means, selection of key blocks.
#include <cmath>
#include <cstring>
#include <type_traits>

#include "../../include/lightcache.h"
#include "lc_internal.h"

namespace lc {
namespace {

lc_status bad(int status, const char* what) { return (lc_status)op_fail(status, "%s", what); }
lc_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LC_OK : (lc_status)op_fail(LC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}
inline bool is_dtype(int dt) { return dt == LC_F32 || dt == LC_BF16; }

// ---- rotary positions ------------------------------------------------------------------------------------------------

struct RopeArgs {
  lc_strides xs, ys;
  int64_t start[3], pos_batch;
  int T, H, axes, pairs, rot, rest;  // rest: channels behind the pairs that are copied (0 in place)
  int pair0[3], dim[3];              // axis a: its first pair, its channels
  int grid1, grid2;                  // cells of the last axes of the grid (1 where there are fewer)
  int tokens;                        // per workgroup
  float amp, sign;
  double turns[LC_ROPE_MAX_PAIRS];
};

template <class T, int N> struct alignas(sizeof(T) * N) Packet { T v[N]; };

// (written out, so that units of any size round alike)
template <class T> __device__ __forceinline__ void turn_pair(T& u, T& v, float c, float s) {
  const float uf = to_f32(u), vf = to_f32(v);
  u = from_f32<T>(fmaf(uf, c, -(vf * s)));
  v = from_f32<T>(fmaf(uf, s, vf * c));
}

// A workgroup turns `tokens` tokens of one batch element. Cosine and sine of a (token, pair) are the same for every head: they are
// formed once, in LDS, and the heads stream past. A thread's unit is VEC pairs of one head: two packets of VEC channels
// (HALF) or one of 2 VEC (interleaved); behind a head's pairs come packets of VEC channels that are copied. Bound by the bytes: 2 x 4096
// tokens, 32 heads of 64, bf16, 13.2 us = 5.1 TB/s (a large copy 5.2); with two or four units of a thread under way at a time 15.0, 13.7.
template <class T, int VEC, bool HALF>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, const T* x, const int32_t* __restrict__ pos, T* y) {
  extern __shared__ __attribute__((aligned(16))) float cs[];  // [token][pair][cos, sin]
  const int b = blockIdx.y, t0 = blockIdx.x * a.tokens, nt = min(a.tokens, a.T - t0);
  const int tid = threadIdx.x;
  for (int i = tid; i < nt * a.pairs; i += 256) {
    const int tt = i / a.pairs, p = i - tt * a.pairs, t = t0 + tt;
    const int ax = (a.axes > 1 && p >= a.pair0[1]) + (a.axes > 2 && p >= a.pair0[2]);
    double at;
    if (pos != nullptr) {
      at = pos[b * a.pos_batch + (int64_t)t * a.axes + ax];
    } else {
      const int c2 = t % a.grid2, r = t / a.grid2;  // one axis: grid1 = grid2 = 1; two: grid1 = 1
      const int cell = a.axes == 1 ? t : ax == a.axes - 1 ? c2 : (a.axes == 3 && ax == 1) ? r % a.grid1 : r / a.grid1;
      at = (double)(a.start[ax] + cell);
    }
    // whole turns go while there are 64 bits: what is left is at most half a turn
    double turn = at * a.turns[p];
    turn -= rint(turn);
    float s, c;
    if constexpr (sizeof(T) == 2) {  // (sine and cosine of turns, off by 2^-20 or so, far below a step of bf16)
      s = __builtin_amdgcn_sinf((float)turn);
      c = __builtin_amdgcn_cosf((float)turn);
    } else {
      sincospif(2.f * (float)turn, &s, &c);
    }
    cs[2 * i] = a.amp * c;
    cs[2 * i + 1] = a.sign * s;
  }
  __syncthreads();
  const int npair = a.pairs / VEC, items = npair + a.rest / VEC, per = 256 / items;
  const int item = tid % items, sub = tid / items;
  if (sub >= per) return;
  const T* const xb = x + b * a.xs.batch;
  T* const yb = y + b * a.ys.batch;
  const int rows = nt * a.H;
  if (item >= npair) {
    typedef Packet<T, VEC> P;
    const int c = a.rot + (item - npair) * VEC;
    for (int r = sub; r < rows; r += per) {
      const int tt = r / a.H, h = r - tt * a.H;
      *reinterpret_cast<P*>(yb + (t0 + tt) * a.ys.token + h * a.ys.head + c) =
          *reinterpret_cast<const P*>(xb + (t0 + tt) * a.xs.token + h * a.xs.head + c);
    }
    return;
  }
  const int p = item * VEC;
  const int ax = (a.axes > 1 && p >= a.pair0[1]) + (a.axes > 2 && p >= a.pair0[2]);
  // the unit's first channel, and with HALF how far its partners are
  const int lo = HALF ? a.pair0[ax] + p : 2 * p, apart = a.dim[ax] / 2;
  for (int r = sub; r < rows; r += per) {
    const int tt = r / a.H, h = r - tt * a.H;
    const float* const w = cs + 2 * (tt * a.pairs + p);
    const T* const xr = xb + (t0 + tt) * a.xs.token + h * a.xs.head + lo;
    T* const yr = yb + (t0 + tt) * a.ys.token + h * a.ys.head + lo;
    if constexpr (HALF) {
      typedef Packet<T, VEC> P;
      P u = *reinterpret_cast<const P*>(xr), v = *reinterpret_cast<const P*>(xr + apart);
#pragma unroll
      for (int e = 0; e < VEC; ++e) turn_pair(u.v[e], v.v[e], w[2 * e], w[2 * e + 1]);
      *reinterpret_cast<P*>(yr) = u;
      *reinterpret_cast<P*>(yr + apart) = v;
    } else {
      typedef Packet<T, 2 * VEC> P;
      P u = *reinterpret_cast<const P*>(xr);
#pragma unroll
      for (int e = 0; e < VEC; ++e) turn_pair(u.v[2 * e], u.v[2 * e + 1], w[2 * e], w[2 * e + 1]);
      *reinterpret_cast<P*>(yr) = u;
    }
  }
}

// every stride and the pointer keep `bytes` alignment
inline bool strides_aligned(const void* p, const lc_strides& s, int dt, size_t bytes) {
  const int64_t es = (int64_t)dtype_size(dt), n = (int64_t)bytes;
  return (uintptr_t)p % bytes == 0 && s.batch * es % n == 0 && s.token * es % n == 0 && s.head * es % n == 0;
}

// ---- block means -----------------------------------------------------------------------------------------------------

// acc += rows r0, r0 + step, .. < n of a packet of channels, eight of them under way at a time (the sums are nothing to the loads). In 64 bits:
// those of 128 bf16 numbers within 2^38 of each other are then exact (8 + 38 + 7 bits).
template <class T>
__device__ __forceinline__ void sum_rows(const T* base, int64_t ld, int r0, int step, int n, double (&acc)[Vec16<T>::N]) {
  constexpr int AHEAD = 8;
  for (int r = r0; r < n; r += AHEAD * step) {
    Vec16<T> v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) v[u] = load16(base + (int64_t)min(r + u * step, n - 1) * ld);
    __builtin_amdgcn_sched_barrier(0);  // (left alone the compiler waits for each where it is added)
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (r + u * step < n) {
#pragma unroll
        for (int e = 0; e < Vec16<T>::N; ++e) acc[e] += (double)v[u].get(e);
      }
  }
}

// A workgroup forms the means of four neighbouring blocks of one (batch element, key head), one a wavefront: its lanes take the
// packets of as many rows at a time as they cover. Bound by the bytes, and by how short its workgroups live: 2 x 4096 keys, 16 heads of 64,
// bf16, 6.3 us for 16.8 MB, 2 x 20011 17.3 us for 67.6 MB (3.9 TB/s).
template <class T>
__global__ __launch_bounds__(256) void block_means_kernel(const T* __restrict__ k, lc_strides ks, const int32_t* __restrict__ k_len,
                                                          double* __restrict__ means, int Tk, int Hkv, int d, int block, int nk,
                                                          int first, int last, int quads) {
  constexpr int VEC = Vec16<T>::N;
  __shared__ double part[4][64 * VEC];
  __shared__ double mean[128][4];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  // (heads first: what neighbouring workgroups read at a time are neighbouring pieces of the same rows)
  const int h = (int)(blockIdx.x % Hkv), bq = (int)(blockIdx.x / Hkv), q4 = bq % quads, b = bq / quads;
  const int j = first + q4 * 4 + wid, len = k_len ? min(max(k_len[b], 0), Tk) : Tk;
  const int t0 = j * block, n = j < last ? min(max(len - t0, 0), block) : 0;
  const int PK = d / VEC, rows = 64 / PK, r0 = lane / PK, pk = lane - r0 * PK;
  double acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.0;
  if (r0 < rows) sum_rows(k + b * ks.batch + h * ks.head + pk * VEC + (int64_t)t0 * ks.token, ks.token, r0, rows, n, acc);
#pragma unroll
  for (int e = 0; e < VEC; ++e) part[wid][lane * VEC + e] = acc[e];
  __syncthreads();
  for (int c = lane; c < d; c += 64) {
    double s = 0.0;
    for (int r = 0; r < rows; ++r) s += part[wid][r * d + c];
    mean[c][wid] = n > 0 ? s / n : 0.0;
  }
  __syncthreads();
  double* const out = means + ((int64_t)b * Hkv + h) * d * nk;
  for (int i = threadIdx.x; i < d * 4; i += 256) {
    const int c = i >> 2, jj = first + q4 * 4 + (i & 3);
    if (jj < last) out[(int64_t)c * nk + jj] = mean[c][i & 3];
  }
}

// ---- selection -------------------------------------------------------------------------------------------------------

struct SelectArgs {
  lc_strides qs;
  const int32_t *q_len, *k_len;
  int64_t q_pos0;
  int Tq, Tk, H, Hkv, d, block, q_block, keep, sink, window, nq, nk, slices;
};

constexpr int kQM = 132;  // doubles from one group's means to the next in LDS: what four groups read at a time lies in different banks

// Scores as unsigned numbers of the same order: 0 no block, 1 a score that is no number, all ones a block that is forced.
__device__ __forceinline__ uint64_t order_of(double s) {
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);  // (-0 is 0)
  if (s != s) return 1;
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// A workgroup of eight wavefronts selects for R neighbouring groups of one (batch element, head). Means of the groups' queries first,
// 8 / R wavefronts a group; then the scores, 16 blocks a wavefront at a time, into LDS as ordered numbers; then a wavefront a group
// searches the keep-th largest of them bit by bit, HELD of them a lane in registers and the rest in LDS, and writes what is not below
// it, by ascending block. Nearly half of the time goes into pooling the queries (2 x 20011 tokens, 313 blocks, 16 heads of 64 34.0 us, 67.6 MB), the rest
// into scores and search; 2 x 4096 tokens, 64 blocks 9.8 us (heads of 16, 32, 40 like those of 64, of 128 13.4). Few queries are a workgroup a head: 4 x 3 against 250
// blocks 10.9 us.
template <class T, int R, int HELD>
__global__ __launch_bounds__(512) void block_select_kernel(SelectArgs a, const T* __restrict__ q, const double* __restrict__ means,
                                                           int32_t* __restrict__ index) {
  constexpr int VEC = Vec16<T>::N, WPR = 8 / R, G4 = (R + 3) / 4;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  double (*const qm)[kQM] = reinterpret_cast<double (*)[kQM]>(smem);      // [R][kQM]
  uint64_t* const keys = reinterpret_cast<uint64_t*>(smem + R * kQM * 8);   // [R][nk]; before that the sums of eight wavefronts
  double* const part = reinterpret_cast<double*>(keys);
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (heads first: as above, and where they are a multiple of eight all groups of a head find its means in one XCD's L2)
  const int h = (int)(blockIdx.x % a.H), bs = (int)(blockIdx.x / a.H), g0 = bs % a.slices * R, b = bs / a.slices;
  const int klen = a.k_len ? min(max(a.k_len[b], 0), a.Tk) : a.Tk, qlen = a.q_len ? min(max(a.q_len[b], 0), a.Tq) : a.Tq;
  const int d = a.d, nk = a.nk, live = (klen + a.block - 1) / a.block;

  {
    const int g = g0 + wid / WPR, PK = d / VEC, rows = 64 / PK, r0 = lane / PK, pk = lane - r0 * PK;
    const int64_t t0 = (int64_t)g * a.q_block;
    const int n = g < a.nq ? (int)min(max((int64_t)qlen - t0, (int64_t)0), (int64_t)a.q_block) : 0;
    double acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.0;
    if (r0 < rows) sum_rows(q + b * a.qs.batch + h * a.qs.head + pk * VEC + t0 * a.qs.token, a.qs.token, r0 + (wid % WPR) * rows, rows * WPR, n, acc);
#pragma unroll
    for (int e = 0; e < VEC; ++e) part[(wid * 64 + lane) * VEC + e] = acc[e];
  }
  __syncthreads();
  for (int i = tid; i < R * d; i += 512) {
    const int r = i / d, c = i - r * d, rows = 64 / (d / VEC);
    const int64_t t0 = (int64_t)(g0 + r) * a.q_block;
    const int n = (int)min(max((int64_t)qlen - t0, (int64_t)0), (int64_t)a.q_block);
    double s = 0.0;
    for (int w = 0; w < WPR; ++w)
      for (int k = 0; k < rows; ++k) s += part[((r * WPR + w) * 64) * VEC + k * d + c];
    qm[r][c] = n > 0 ? s / n : 0.0;
  }
  __syncthreads();

  // Scores of 16 blocks at a time on the matrix cores: four 4 x 4 x 4 products side by side, whose rows are four groups and whose 16 columns
  // are the blocks. (A lane a block and fused multiply-adds, whose every score reads its group's mean out of LDS, take 19.7 us in place of 14.4 at
  // 2 x 8192 tokens.)
  const double* const mb = means + ((int64_t)b * a.Hkv + h / (a.H / a.Hkv)) * d * nk;
  {
    const int kq = lane >> 4;
    const double* const qa = &qm[(lane & 3) % R][kq];
    for (int j = wid * 16 + (lane & 15); j - (lane & 15) < live; j += 8 * 16) {
      const double* const mj = mb + (int64_t)kq * nk + min(j, nk - 1);  // (behind the last block it stands in: nothing of it is kept)
      double s[G4];
#pragma unroll
      for (int u = 0; u < G4; ++u) s[u] = 0.0;
      auto batch = [&](int c0, auto n_c) {
        constexpr int N = decltype(n_c)::value;
        double m[N];
#pragma unroll
        for (int c = 0; c < N; ++c) m[c] = mj[(int64_t)(c0 + 4 * c) * nk];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
          for (int u = 0; u < G4; ++u)
            s[u] = __builtin_amdgcn_mfma_f64_4x4x4f64(qa[u * 4 * kQM + c0 + 4 * c], m[c], s[u], 0, 0, 0);
      };
      int c0 = 0;
      for (; c0 + 64 <= d; c0 += 64) batch(c0, std::integral_constant<int, 16>{});
      for (; c0 < d; c0 += 8) batch(c0, std::integral_constant<int, 2>{});
#pragma unroll
      for (int u = 0; u < G4; ++u) {
        const int r = u * 4 + kq;
        const int64_t p0 = a.q_pos0 + (int64_t)(g0 + r) * a.q_block, p1 = min(p0 + a.q_block, a.q_pos0 + qlen) - 1;  // (of queries that exist)
        const bool near = a.window >= 0 && ((int64_t)j - a.window) * a.block <= p1 &&
                          ((int64_t)j + a.window + 1) * a.block > p0;  // (both say what a floor would, below zero too)
        if (r < R && j < live) keys[r * nk + j] = j < a.sink || near ? ~0ull : order_of(s[u]);
      }
    }
  }
  __syncthreads();

  if (wid >= R || g0 + wid >= a.nq) return;
  const int g = g0 + wid;
  const uint64_t* const kr = keys + wid * nk;
  int32_t* const out = index + (((int64_t)b * a.H + h) * a.nq + g) * a.keep;
  int written = 0;
  if ((int64_t)g * a.q_block < qlen) {
    const int chunks = (live + 63) / 64;
    uint64_t held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = i * 64 + lane < live ? kr[i * 64 + lane] : 0;
    auto count = [&](uint64_t least) {  // blocks whose number is at least that (not 0: lanes without a block hold it)
      int n = 0;
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        n += __popcll(__builtin_amdgcn_ballot_w64(held[i] >= least));
      for (int i = HELD; i < chunks; ++i)
        n += __popcll(__builtin_amdgcn_ballot_w64(i * 64 + lane < live && kr[i * 64 + lane] >= least));
      return n;
    };
    auto count_upper = [&](uint32_t least) {  // the same of the upper halves (not 0)
      int n = 0;
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        n += __popcll(__builtin_amdgcn_ballot_w64((uint32_t)(held[i] >> 32) >= least));
      for (int i = HELD; i < chunks; ++i)
        n += __popcll(__builtin_amdgcn_ballot_w64(i * 64 + lane < live && (uint32_t)(kr[i * 64 + lane] >> 32) >= least));
      return n;
    };
    // What is listed: numbers above `least`, and the first `ties` of those that equal it. Forced blocks and scores that are no
    // numbers are counted at the ends; among the others the bits that all have in common need no search.
    uint64_t least = 1;
    int ties = live;
    if (live > a.keep) {
      const int forced = count(~0ull), real = count(2) - forced, want = a.keep - forced;
      if (want <= 0) {
        least = ~0ull;
        ties = a.keep;
      } else if (real <= want) {
        ties = want - real;
      } else {
        uint64_t all = ~0ull, any = 0;
        auto look = [&](uint64_t v) {
          if (v > 1 && v != ~0ull) {
            all &= v;
            any |= v;
          }
        };
#pragma unroll
        for (int i = 0; i < HELD; ++i) look(held[i]);
        for (int i = HELD; i < chunks; ++i) look(i * 64 + lane < live ? kr[i * 64 + lane] : 0);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          all &= (uint64_t)__shfl_xor((long long)all, o, 64);
          any |= (uint64_t)__shfl_xor((long long)any, o, 64);
        }
        least = all;
        ties = want;  // (all of them equal: the first ones)
        if (all != any) {
          int bit = 63 - __builtin_clzll(all ^ any), n = 0;
          least = any >> bit >> 1 << bit << 1;
          for (; bit >= 32 && n != a.keep; --bit) {  // (the upper halves nearly always tell)
            const uint64_t more = least | 1ull << bit;
            n = count_upper((uint32_t)(more >> 32));
            if (n >= a.keep) least = more;
          }
          for (; bit >= 0 && n != a.keep; --bit) {
            const uint64_t more = least | 1ull << bit;
            n = count(more);
            if (n >= a.keep) least = more;
          }
          ties = a.keep - count(least + 1);
        }
      }
    }
    for (int i = 0; i < chunks; ++i) {
      const int j = i * 64 + lane;
      const uint64_t v = j < live ? kr[j] : 0;
      const uint64_t below = (1ull << lane) - 1;
      const bool tie = j < live && v == least;
      const uint64_t tb = __builtin_amdgcn_ballot_w64(tie);
      const bool take = (j < live && v > least) || (tie && __popcll(tb & below) < ties);
      const uint64_t kb = __builtin_amdgcn_ballot_w64(take);
      if (take) out[written + __popcll(kb & below)] = j;
      ties -= min(ties, __popcll(tb));
      written += __popcll(kb);
    }
  }
  for (int i = written + lane; i < a.keep; i += 64) out[i] = -1;
}

}  // namespace

// shared with lc_battn.hip: what all calls of the sparse operators require of their descriptor
int check_sparse_args(const lc_sparse_args* a) {
  if (!a) return bad(LC_ERR_ARG, "args is NULL");
  if (!is_dtype(a->dtype)) return bad(LC_ERR_ARG, "dtype must be LC_F32 or LC_BF16");
  if (a->B <= 0 || a->Tq <= 0 || a->Tk <= 0 || a->heads <= 0 || a->kv_heads <= 0) return bad(LC_ERR_SHAPE, "all sizes must be positive");
  if (a->heads % a->kv_heads) return bad(LC_ERR_SHAPE, "heads must be a multiple of kv_heads");
  const int d = a->head_dim;
  if (!(d == 8 || d == 16 || d == 32 || d == 40 || d == 64 || d == 128)) return bad(LC_ERR_SHAPE, "head_dim must be one of 8, 16, 32, 40, 64, 128");
  if (a->block <= 0 || a->block % 64) return bad(LC_ERR_SHAPE, "block must be a positive multiple of 64");
  if (a->q_block < 1 || a->q_block > 128) return bad(LC_ERR_SHAPE, "q_block must be in [1, 128]");
  if (a->keep < 1 || a->keep > 65536) return bad(LC_ERR_SHAPE, "keep must be in [1, 65536]");
  if (a->Tk > 1 << 30 || a->block > 1 << 20) return bad(LC_ERR_SHAPE, "Tk must be at most 2^30 and block at most 2^20");
  if (((int64_t)a->Tk + a->block - 1) / a->block > 8192) return bad(LC_ERR_SHAPE, "more than 8192 key blocks: use larger ones");
  if ((int64_t)a->B * a->heads > 1 << 24) return bad(LC_ERR_SHAPE, "at most 2^24 heads of all batch elements");
  return LC_OK;
}
// an output: no axis of stride zero
bool strides_apart(const lc_strides& s, int B, int T, int heads) {
  return (B == 1 || s.batch != 0) && (T == 1 || s.token != 0) && (heads == 1 || s.head != 0);
}
// one strided input or output whose rows are moved in 16-byte packets
int check_sparse_rows(const char* name, const void* p, const lc_strides& s, int dt) {
  if (!p) return op_fail(LC_ERR_ARG, "%s is NULL", name);
  if (!strides_aligned(p, s, dt, 16)) return op_fail(LC_ERR_SHAPE, "every head's row of %s must be 16-byte aligned", name);
  return LC_OK;
}

}  // namespace lc

using namespace lc;

extern "C" {

lc_status lc_rope_make(const lc_rope_config* g, lc_rope_table* out) {
  if (!g || !out) return bad(LC_ERR_ARG, "cfg and out must not be NULL");
  if (g->head_dim < 2 || g->head_dim > 2 * LC_ROPE_MAX_PAIRS) return bad(LC_ERR_SHAPE, "head_dim must be in [2, 128]");
  if (g->axes < 1 || g->axes > 3) return bad(LC_ERR_SHAPE, "axes must be in [1, 3]");
  if (g->layout != LC_ROPE_HALF && g->layout != LC_ROPE_INTERLEAVED) return bad(LC_ERR_ARG, "layout must be LC_ROPE_HALF or LC_ROPE_INTERLEAVED");
  if (g->scaling < LC_ROPE_UNSCALED || g->scaling > LC_ROPE_PARTS) return bad(LC_ERR_ARG, "scaling must be one of LC_ROPE_UNSCALED .. LC_ROPE_PARTS");
  if (!(g->base > 1.0) || !std::isfinite(g->base)) return bad(LC_ERR_SHAPE, "base must be greater than 1");
  if (g->scaling != LC_ROPE_UNSCALED && (!(g->factor > 0.0) || !std::isfinite(g->factor))) return bad(LC_ERR_SHAPE, "factor must be positive");
  if (g->scaling == LC_ROPE_PARTS && (g->orig_len <= 0 || !(g->beta_fast > g->beta_slow) || !std::isfinite(g->beta_fast) || !std::isfinite(g->beta_slow)))
    return bad(LC_ERR_SHAPE, "orig_len must be positive and beta_fast greater than beta_slow");
  int rot = 0;
  for (int a = 0; a < g->axes; ++a) {
    if (g->axis_dim[a] <= 0 || g->axis_dim[a] % 2 || g->axis_dim[a] > g->head_dim) return bad(LC_ERR_SHAPE, "axis_dim must be even, positive and at most head_dim");
    rot += g->axis_dim[a];
  }
  if (rot > g->head_dim) return bad(LC_ERR_SHAPE, "the axes take more channels than head_dim");
  lc_rope_table t;
  memset(&t, 0, sizeof t);
  t.head_dim = g->head_dim; t.rot_dim = rot; t.axes = g->axes; t.layout = g->layout;
  t.amplitude = g->scaling == LC_ROPE_PARTS && g->factor > 1.0 ? 0.1 * std::log(g->factor) + 1.0 : 1.0;
  const double two_pi = 6.283185307179586476925286766559;
  const double kFastest = 18446744073709551616.0;  // (such angles have long lost their precision, and end in infinities)
  int n = 0;
  for (int a = 0; a < g->axes; ++a) {
    const int D = g->axis_dim[a];
    t.axis_dim[a] = D;
    const double base = g->scaling == LC_ROPE_BASE && D > 2 ? g->base * std::pow(g->factor, (double)D / (D - 2)) : g->base;
    if (!(base > 0.0) || !std::isfinite(base)) return bad(LC_ERR_SHAPE, "factor takes the base out of the range of 64 bits");
    for (int i = 0; i < D / 2; ++i) {
      double w = std::pow(base, -2.0 * i / D);
      if (g->scaling == LC_ROPE_LINEAR) w /= g->factor;
      if (g->scaling == LC_ROPE_PARTS) {
        double keep = (g->orig_len * w / two_pi - g->beta_slow) / (g->beta_fast - g->beta_slow);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        w = w * (keep + (1.0 - keep) / g->factor);
      }
      if (!(w <= kFastest)) return bad(LC_ERR_SHAPE, "factor makes a pair turn more than 2^64 radians a position");
      t.turns[n++] = w / two_pi;
    }
  }
  t.checked = 1;
  *out = t;
  return LC_OK;
}

lc_status lc_op_rope(const lc_rope_table* t, const lc_rope_args* a, const void* x, const int32_t* pos, void* y, void* stream) {
  if (!t || !a || !x || !y) return bad(LC_ERR_ARG, "table, args, x and y must not be NULL");
  if (t->checked != 1 || t->axes < 1 || t->axes > 3 || t->rot_dim < 2 || t->rot_dim > t->head_dim || t->head_dim > 2 * LC_ROPE_MAX_PAIRS)
    return bad(LC_ERR_ARG, "table was not made by lc_rope_make");
  if (!is_dtype(a->dtype)) return bad(LC_ERR_ARG, "dtype must be LC_F32 or LC_BF16");
  if (a->B <= 0 || a->T <= 0 || a->heads <= 0) return bad(LC_ERR_SHAPE, "all sizes must be positive");
  if (a->inverse != 0 && a->inverse != 1) return bad(LC_ERR_ARG, "inverse must be 0 or 1");
  if (a->heads > 1 << 20 || a->T > 1 << 27) return bad(LC_ERR_SHAPE, "at most 2^20 heads and 2^27 tokens");
  if (!strides_apart(a->y, a->B, a->T, a->heads)) return bad(LC_ERR_SHAPE, "the rows of y must not overlap");
  RopeArgs k;
  k.xs = a->x; k.ys = a->y;
  k.T = a->T; k.H = a->heads; k.axes = t->axes; k.pairs = t->rot_dim / 2; k.rot = t->rot_dim;
  k.grid1 = k.grid2 = 1;
  k.pos_batch = a->pos_batch;
  int n = 0;
  for (int i = 0; i < 3; ++i) {
    k.pair0[i] = n;
    k.dim[i] = i < t->axes ? t->axis_dim[i] : 0;
    if (k.dim[i] < 0 || k.dim[i] % 2) return bad(LC_ERR_ARG, "table was not made by lc_rope_make");
    n += k.dim[i] / 2;
    k.start[i] = a->start[i];
  }
  if (n != k.pairs) return bad(LC_ERR_ARG, "table was not made by lc_rope_make");
  if (!pos) {
    for (int i = 0; i < t->axes; ++i)
      if (a->start[i] > (int64_t)1 << 40 || a->start[i] < -((int64_t)1 << 40)) return bad(LC_ERR_SHAPE, "start must be within 2^40");
    for (int i = 1; i < t->axes; ++i)
      if (a->grid[i] <= 0) return bad(LC_ERR_SHAPE, "positions on several axes need pos or a grid");
    if (t->axes > 1) k.grid2 = a->grid[t->axes - 1];
    if (t->axes > 2) k.grid1 = a->grid[1];
  }
  const bool in_place = x == y;
  if (in_place && memcmp(&a->x, &a->y, sizeof a->x)) return bad(LC_ERR_SHAPE, "in place, x and y have the same strides");
  k.rest = in_place ? 0 : t->head_dim - t->rot_dim;
  k.amp = (float)t->amplitude;
  k.sign = a->inverse ? -k.amp : k.amp;
  memcpy(k.turns, t->turns, sizeof k.turns);
  if (a->B > 65535) return bad(LC_ERR_SHAPE, "B must be at most 65535");
  const int es = (int)dtype_size(a->dtype);
  auto fits = [&](int vec) {  // units of vec pairs: whole and aligned
    const size_t bytes = (size_t)(t->layout == LC_ROPE_HALF ? vec : 2 * vec) * es;
    if (k.rest % vec || !strides_aligned(x, a->x, a->dtype, bytes) || !strides_aligned(y, a->y, a->dtype, bytes)) return false;
    for (int i = 0; i < t->axes; ++i)
      if (k.dim[i] / 2 % vec) return false;
    return true;
  };
  // (us, 2 x 4096 tokens of 2048 channels: heads of 128 in axes of 44, 42, 42, which move channel by channel, against heads of 64 in axes of 16, 24, 24: bf16
  // half 25.4 and 14.2, interleaved 23.1 and 13.4; float half 36.0 and 30.8, interleaved 33.4 and 29.5)
  const bool half = t->layout == LC_ROPE_HALF, bf = a->dtype == LC_BF16;
  const int vec = half && bf && fits(8) ? 8 : (half || bf) && fits(4) ? 4 : !half && !bf && fits(2) ? 2 : 1;
  // Tokens a workgroup: some 1024 units, four a thread, so that the trigonometry is shared out and few workgroups start (32 heads of 64: 4
  // tokens 13.7 us, one 17.7; 16 heads: 8 tokens 29.5 us of 123 MB, one 53.6), as long as there are two for each compute unit (1000
  // tokens of 32 heads: one 5.3 us, 8 a workgroup 6.6). A launch counts its threads in 32 bits: 2^24 tokens and more are two at least.
  const int units = a->heads * (k.pairs / vec + k.rest / vec);
  k.tokens = 1;
  while ((a->T + k.tokens - 1) / k.tokens >= 1 << 24) k.tokens *= 2;
  while (k.tokens < 64 && 2 * k.tokens * (int64_t)units <= 1024 && (int64_t)a->B * ((a->T + 2 * k.tokens - 1) / (2 * k.tokens)) >= 512) k.tokens *= 2;
  const dim3 grid((unsigned)((a->T + k.tokens - 1) / k.tokens), (unsigned)a->B);
  const size_t lds = (size_t)k.tokens * k.pairs * 8;
#define LC_GO(T, V, HALF) rope_kernel<T, V, HALF><<<grid, 256, lds, (hipStream_t)stream>>>(k, (const T*)x, pos, (T*)y)
  if (bf && half) {
    if (vec == 8) LC_GO(bf16_t, 8, true); else if (vec == 4) LC_GO(bf16_t, 4, true); else LC_GO(bf16_t, 1, true);
  } else if (bf) {
    if (vec == 4) LC_GO(bf16_t, 4, false); else LC_GO(bf16_t, 1, false);
  } else if (half) {
    if (vec == 4) LC_GO(float, 4, true); else LC_GO(float, 1, true);
  } else {
    if (vec == 2) LC_GO(float, 2, false); else LC_GO(float, 1, false);
  }
#undef LC_GO
  return launched("rope");
}

int32_t lc_sparse_groups(const lc_sparse_args* a) {
  return a && a->Tq > 0 && a->q_block > 0 ? (int32_t)(((int64_t)a->Tq + a->q_block - 1) / a->q_block) : 0;
}
int32_t lc_sparse_blocks(const lc_sparse_args* a) {
  return a && a->Tk > 0 && a->block > 0 ? (int32_t)(((int64_t)a->Tk + a->block - 1) / a->block) : 0;
}

lc_status lc_op_block_means(const lc_sparse_args* a, const void* k, const int32_t* k_len, double* means, int first, int count, void* stream) {
  int s = check_sparse_args(a);
  if (s == LC_OK) s = check_sparse_rows("k", k, a->k, a->dtype);
  if (s != LC_OK) return (lc_status)s;
  if (!means) return bad(LC_ERR_ARG, "means is NULL");
  const int nk = lc_sparse_blocks(a);
  if (first < 0 || count < 0 || count > nk || first > nk - count) return bad(LC_ERR_ARG, "blocks out of range");
  if (count == 0) return LC_OK;
  const int quads = (count + 3) / 4;
  const int64_t blocks = (int64_t)quads * a->kv_heads * a->B;
  if (blocks > (int64_t)1 << 23) return bad(LC_ERR_SHAPE, "too many blocks");
#define LC_GO(T)                                                                                                                      \
  block_means_kernel<T><<<(unsigned)blocks, 256, 0, (hipStream_t)stream>>>((const T*)k, a->k, k_len, means, a->Tk, a->kv_heads, a->head_dim, \
                                                                           a->block, nk, first, first + count, quads)
  if (a->dtype == LC_BF16) LC_GO(bf16_t); else LC_GO(float);
#undef LC_GO
  return launched("block_means");
}

lc_status lc_op_block_select(const lc_sparse_args* a, const void* q, const double* means, const int32_t* q_len, const int32_t* k_len,
                             int32_t* index, void* stream) {
  int s = check_sparse_args(a);
  if (s == LC_OK) s = check_sparse_rows("q", q, a->q, a->dtype);
  if (s != LC_OK) return (lc_status)s;
  if (!means || !index) return bad(LC_ERR_ARG, "means and index must not be NULL");
  if (a->sink < 0) return bad(LC_ERR_ARG, "sink must not be negative");
  if (a->q_pos0 > (int64_t)1 << 40 || a->q_pos0 < -((int64_t)1 << 40)) return bad(LC_ERR_SHAPE, "q_pos0 must be within 2^40");
  SelectArgs k;
  k.qs = a->q; k.q_len = q_len; k.k_len = k_len; k.q_pos0 = a->q_pos0;
  k.Tq = a->Tq; k.Tk = a->Tk; k.H = a->heads; k.Hkv = a->kv_heads; k.d = a->head_dim; k.block = a->block; k.q_block = a->q_block;
  k.keep = a->keep; k.sink = a->sink; k.window = a->window; k.nq = lc_sparse_groups(a); k.nk = lc_sparse_blocks(a);
  // Groups a workgroup: as many as share the means best while there is a workgroup for each compute unit, and while the
  // scores' numbers fit into 64 KiB (us with 256 workgroups at least, and with 512: 2 x 4096 tokens 9.8 and 10.2, 1 x 4096 8.6 and 9.7, 2 x 8192 14.0 and 14.4,
  // 1 x 12000 15.1 and 16.9; with 128: 10.7, 8.7, 13.7, 15.5)
  const int64_t bh = (int64_t)a->B * a->heads;
  int R = 8;
  while (R > 1 && (bh * ((k.nq + R - 1) / R) < 256 || R * (k.nk + kQM) > 8192)) R /= 2;
  k.slices = (k.nq + R - 1) / R;
  const int64_t blocks = bh * k.slices;
  if (blocks > (int64_t)1 << 22) return bad(LC_ERR_SHAPE, "too many groups of queries");
  const size_t sums = (size_t)8 * 64 * (a->dtype == LC_BF16 ? 8 : 4) * 8, nums = (size_t)R * k.nk * 8;
  const size_t lds = (size_t)R * kQM * 8 + (sums > nums ? sums : nums);
#define LC_RUN(T, R_, N_)                                                                                                          \
  do {                                                                                                                             \
    const hipError_t e = lds <= 65536 ? hipSuccess : hipFuncSetAttribute((const void*)block_select_kernel<T, R_, N_>,              \
                                                                         hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);    \
    if (e != hipSuccess) return (lc_status)op_fail(LC_ERR_HIP, "block_select: %s", hipGetErrorString(e));                          \
    block_select_kernel<T, R_, N_><<<(unsigned)blocks, 512, lds, (hipStream_t)stream>>>(k, (const T*)q, means, index);             \
  } while (0)
#define LC_GO(R_, N_) do { if (a->dtype == LC_BF16) LC_RUN(bf16_t, R_, N_); else LC_RUN(float, R_, N_); } while (0)
  // (as many held as there are, where that is few: 313 blocks 35.3 us with five, 36.9 with eight)
#define LC_HELD(R_) do { if (chunks > 5) LC_GO(R_, 8); else if (chunks > 2) LC_GO(R_, 5); else if (chunks > 1) LC_GO(R_, 2); else LC_GO(R_, 1); } while (0)
  const int chunks = (k.nk + 63) / 64;
  if (R == 8) LC_HELD(8); else if (R == 4) LC_HELD(4); else if (R == 2) LC_HELD(2); else LC_HELD(1);
#undef LC_HELD
#undef LC_GO
#undef LC_RUN
  return launched("block_select");
}

}  // extern "C"
