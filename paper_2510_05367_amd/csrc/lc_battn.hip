// Attention over listed key blocks.
//
// A workgroup owns one group of queries of one (batch element, head) and walks the 64-key chunks of the blocks that the
// group has listed, keeping per query the running maximum and sum of its softmax, so that no score leaves the registers. Scores are
// formed transposed, S^T[key][query] = K Q^T in 32 x 32 tiles: a lane then holds 16 keys of one query, the statistics are in-lane
// but for one exchange, and the probabilities, rounded to the operands' type, are the B operand of O^T[dim][query] += V^T P^T as they
// are (the matrix instruction takes no others; the denominator sums the same rounded numbers, and bf16 outputs of randomly drawn inputs are
// off by 2.3e-3 of their norm where a float computation that rounds its result alone is off by 1.6e-3). K and V rows go from memory straight into LDS, 16 bytes a lane, through buffer descriptors whose range check
// delivers zeros for the keys beyond the sequence; the transposed V operand is read out of the rows with the
// transposing LDS read (bf16), so no transposed copy of V exists anywhere.
//
// What bounds it in large calls is the vector unit (active 67 % of the cycles) beside the matrix pipe (47 %), and a clock that falls to 1.83 GHz: 33001
// tokens, 16 heads of 64, 64 of 516 blocks 598 us = 925 TFLOP/s (a large matrix product 1226). At 609 us, half the LDS reads left out changed
// nothing, and leaving out the exponentials gave 530. Small calls are 10 us of launch, dependent loads and first bytes, and 2.2 us a listed block at 2 x 4096
// tokens (985 TFLOP/s). With prescaled queries out of packed rows, as the transformer stack calls it, 562 and 45.0 us where dense unscaled ones take 600 and 46.5
// (medians of calls in turn).
#include <atomic>

#include "../../include/lightcache.h"
#include "lc_internal.h"

namespace lc {

int check_sparse_args(const lc_sparse_args* a);  // lc_tokens.hip
int check_sparse_rows(const char* name, const void* p, const lc_strides& s, int dt);
bool strides_apart(const lc_strides& s, int B, int T, int heads);

namespace {

typedef __attribute__((address_space(3))) unsigned char* lds_ptr;
typedef __attribute__((ext_vector_type(4))) short s16x4;

// Division of numbers below 2^31 by one that the host knows: a multiplication (the compiler's division is some thirty
// instructions, and a workgroup finds its place with seven of them)
struct Div {
  uint32_t d, m, s;
  Div() = default;
  explicit Div(int64_t by) : d((uint32_t)by), s(0) {
    while (s < 31 && (1u << s) < d) ++s;
    m = (uint32_t)((((uint64_t)1 << 32) * ((1u << s) - d)) / d + 1);
  }
  __device__ __forceinline__ uint32_t quot(uint32_t n) const { return (uint32_t)(((uint64_t)__umulhi(m, n) + n) >> s); }
};

struct BlockAttnArgs {
  Div per_run, per_prob, by_splits, by_parts, by_H, by_group;  // workgroups of `unit` heads, of one; .. heads that share a key head
  lc_strides qs, ks, vs, os;
  const int32_t *index, *q_len, *k_len;
  float* part;      // several workgroups a list: [query of all][split][D] sums, then [query of all][split][2] maxima and denominators
  float scale;      // of a score, to log2 units
  int B, Tq, Tk, H, Hkv, block, q_block, keep, nq;
  int parts, splits; // workgroups of a group: for 128 / KS of its queries each, and for a share of its list each
  int unit;         // heads in a row that go to one XCD (0: workgroups are dealt out as they come)
};

// KS: wavefronts that share a tile of 32 queries and take turns at its keys. 1: four tiles (groups of up to 128 queries), every
// wavefront takes all keys; 2: two tiles, 32 of the 64 keys of a chunk each; 4: one tile, and two chunks at a time. (Two tiles a
// wavefront halve the fragment reads, but leave room for two wavefronts a SIMD in place of four: 16 heads of 64, 16 of 64 blocks,
// 2 x 4096 tokens 51 and 56 us, groups of 64 queries 56 and 69; LDS is not what bounds this.)
template <class T, int D, int KS> struct BlockAttnShape {
  static constexpr int VEC = Vec16<T>::N;
  static constexpr int PK = D / VEC;             // 16-byte packets of a row
  static constexpr int KP = (PK + 1) / 2 * 2;    // ... in LDS, those beyond D being zeros
  static constexpr int DM = (D + 31) / 32;       // 32-row tiles of O^T
  static constexpr int TILE = 64 * KP * 16;      // bytes of a chunk's K rows, or of its V rows
  static constexpr int NCH = KS == 4 && 2 * TILE <= 32768 ? 2 : 1;  // chunks of a stage
  static constexpr int STAGE = NCH * 2 * TILE;
  static constexpr int NB = 2;                   // stages in LDS
  static constexpr int HAND = (DM * 16 + 2) * 64 * 4;  // what a wavefront hands to another at the end
  static constexpr int RED = KS == 1 ? 0 : 2 * HAND;
  static constexpr int LDS = NB * STAGE > RED ? NB * STAGE : RED;
  static constexpr int LPW = NCH * KP / 2;       // loads of a stage that a wavefront issues
};

// PRE: the queries hold Q log2(e) / sqrt(D). The scores' sums then start from what the exponents subtract, and the exponential takes them as
// they come (2 x 4096 tokens, 16 of 64 blocks 51.2 -> 48.6 us; 33001 tokens, 64 of 516 blocks 610 -> 577).
template <class T, int D, int KS, bool PRE>
__global__ __launch_bounds__(256, 2) void block_attn_kernel(BlockAttnArgs a, const T* __restrict__ q, const T* __restrict__ k,
                                                            const T* __restrict__ v, T* __restrict__ out) {
  typedef BlockAttnShape<T, D, KS> S;
  typedef Mma32<T> M;
  constexpr int VEC = S::VEC, PK = S::PK, KP = S::KP, DM = S::DM, NCH = S::NCH, NB = S::NB, LPW = S::LPW;
  constexpr int KT = KS == 1 ? 2 : 1;      // 32-key sub-tiles of a stage and wavefront
  constexpr int STEPS = KP / 2;            // packets a lane contracts along d
  constexpr bool BF = sizeof(T) == 2;
  constexpr bool kPrio = BF && D <= 64;
  constexpr bool POW2 = (KP & (KP - 1)) == 0;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, hh = lane >> 5;
  // Workgroups are handed to the XCDs in turn: all that read the same keys and values (the groups of a head, and the heads that
  // share it) are put on one, whose L2 then fetches them once
  uint32_t prob, in = blockIdx.x;
  if (a.unit > 0) {
    const uint32_t slot = in >> 3, u8 = a.per_run.quot(slot), w = slot - u8 * a.per_run.d, p = a.per_prob.quot(w);
    prob = ((in & 7) + 8 * u8) * a.unit + p;
    in = w - p * a.per_prob.d;
  } else {
    prob = a.per_prob.quot(in);
    in -= prob * a.per_prob.d;
  }
  const int gp = (int)a.by_splits.quot(in), split = (int)in - gp * a.splits, g = (int)a.by_parts.quot(gp), part = gp - g * a.parts;
  const int b = (int)a.by_H.quot(prob), h = (int)prob - b * a.H, hk = (int)a.by_group.quot(h);
  const int32_t* const list = a.index + ((int64_t)prob * a.nq + g) * a.keep;
  int ent = list[min(lane, a.keep - 1)];  // a lane holds an entry of the list, 64 at a time
  const int row0 = g * a.q_block + part * (128 / KS);            // first query
  const int most = min(a.Tq - row0, min(a.q_block - part * (128 / KS), 128 / KS));  // and how many there could be

  // ---- queries: B operand of S^T = K Q^T; packets beyond D and rows beyond the group are zeros. (Rows behind q_len may hold anything: a
  // query's column of everything below is its own, and theirs are not stored. Were the length waited for, 4 x 3 queries would take 10.2 us
  // in place of 8.6, without lengths too.)
  const int qi = wid / KS * 32 + lq;
  Vec16<T> qf[STEPS];
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const int pk = 2 * j + hh;
    qf[j] = qi < most && pk < PK ? load16(q + b * a.qs.batch + (int64_t)(row0 + qi) * a.qs.token + h * a.qs.head + pk * VEC) : zero16<T>();
  }

  const int TK = a.k_len ? min(max(a.k_len[b], 0), a.Tk) : a.Tk;
  const int rows = a.q_len ? min(most, a.q_len[b] - row0) : most;
  if (rows <= 0) return;

  // the list ends before its first entry that is no existing block or does not ascend
  int n = a.keep;
  for (int i0 = 0, last = -1; i0 < a.keep; i0 += 64) {
    const int e = i0 == 0 ? ent : list[min(i0 + lane, a.keep - 1)];
    const int prev = __shfl_up(e, 1, 64);
    const bool bad = i0 + lane < a.keep && (e < 0 || (int64_t)e * a.block >= TK || e <= (lane == 0 ? last : prev));
    const uint64_t bads = __builtin_amdgcn_ballot_w64(bad);
    if (bads != 0) {
      n = i0 + __builtin_ctzll(bads);
      break;
    }
    last = __builtin_amdgcn_readlane(e, 63);
  }
  const int cpb = a.block / 64, chunks = __builtin_amdgcn_readfirstlane(n) * cpb;
  const int c_lo = (int)((int64_t)chunks * split / a.splits), c_hi = (int)((int64_t)chunks * (split + 1) / a.splits);
  const int nstage = (c_hi - c_lo + NCH - 1) / NCH;

  // ---- what this wavefront moves: K or V rows of one chunk of a stage, or half of them
  const int my_chunk = NCH == 2 ? wid >> 1 : 0;
  const bool moves_v = NCH == 2 ? wid & 1 : wid >> 1;
  const int first = NCH == 2 ? 0 : (wid & 1) * LPW;  // load of the tile
  const int64_t ld = moves_v ? a.vs.token : a.ks.token;
  const T* const src = moves_v ? v + b * a.vs.batch + hk * a.vs.head : k + b * a.ks.batch + hk * a.ks.head;
  // 16-byte slots are swizzled so that what neighbouring lanes read together lies in different banks: K rows are read a
  // slot of 32 rows at a time, V rows 64 bytes of four rows (bf16), or 128 bytes of a row and of the fourth behind it (float)
  auto k_swz = [](int key) { return !POW2 ? 0 : KP >= 16 ? key & 15 : (key / (16 / KP)) & (KP - 1); };
  auto v_swz = [](int key) {
    if (BF) return KP == 8 ? ((key >> 1) & 1) * 4 : KP == 16 ? (key & 3) * 4 : 0;
    return KP >= 16 ? ((key >> 2) & 1) * 8 : 0;
  };
  uint32_t off[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int p = (first + i) * 64 + lane, key = p / KP, c = (p - key * KP) ^ (moves_v ? v_swz(key) : k_swz(key));
    off[i] = c < PK ? (uint32_t)(key * ld + c * VEC) * (uint32_t)sizeof(T) : 0x7fffff00u;
  }
  const unsigned lds_at = (my_chunk * 2 + (moves_v ? 1 : 0)) * S::TILE + first * 1024;
  // The chunks of the list in turn, TK (no keys) behind the end
  int at = c_lo + my_chunk, at_li = at / cpb, at_sub = at - at_li * cpb, held = 0;
  auto next_key0 = [&]() {
    if (at >= c_hi) return TK;
    if (at_li - held >= 64) {
      held = at_li & ~63;
      ent = list[min(held + lane, a.keep - 1)];
      asm volatile("" : "+v"(ent));
    }
    const int key0 = __builtin_amdgcn_readlane(ent, at_li & 63) * a.block + at_sub * 64;
    at += NCH;
    at_sub += NCH;
    while (at_sub >= cpb) {
      at_sub -= cpb;
      ++at_li;
    }
    return key0;
  };
  // The requests are written out, so that the compiler does not take the transposing reads below to depend on all of them and
  // waits for none: barrier_keep says when a stage is there. (No register is loaded. The wait states in front are what a load needs behind
  // vector instructions that wrote its scalar operands. m0, where the load finds its place in LDS, is reserved: the compiler warns of it in a clobber
  // list and uses it for nothing else here, which a test of the compiled code holds it to.)
  auto issue = [&](int st, int key0) {
#ifdef __HIP_DEVICE_COMPILE__
    const int keys = min(64, TK - key0);
    const uint64_t base = (uint64_t)(src + key0 * ld);
    typedef __attribute__((ext_vector_type(4))) int i32x4;
    i32x4 r = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)((uint32_t)(base >> 32) & 0xffffu)),
                     __builtin_amdgcn_readfirstlane(keys > 0 ? (int)(((keys - 1) * ld + D) * (int)sizeof(T)) : 0), 0x00020000};  // (raw 32-bit data)
    uint32_t dst = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)(smem + (st % NB) * S::STAGE + lds_at));
    asm volatile("s_nop 4" : "+s"(r), "+s"(dst)::"memory");
#pragma unroll
    for (int i = 0; i < LPW; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst + i * 1024), "v"(off[i]), "s"(r) : "memory");
#else
    (void)st; (void)key0; (void)off; (void)lds_at; (void)src;
#endif
  };

  const int half = KS == 1 ? 0 : wid & 1;          // of the chunk
  const bool busy = KS != 4 || (wid >> 1) < NCH;   // (one chunk a stage leaves two of four wavefronts without keys)
  const unsigned k_at = my_chunk * 2 * S::TILE + lq * (KP * 16), v_at = (my_chunk * 2 + 1) * S::TILE;
  unsigned v_off[DM];
  const int trow = BF ? (lane & 15) >> 2 : 0;
#pragma unroll
  for (int mt = 0; mt < DM; ++mt) {
    if constexpr (BF) {  // 16 lanes read 16 dims of four keys: lane i four dims of key i / 4
      const int dim = mt * 32 + ((lane >> 4) & 1) * 16 + 4 * (lane & 3), slot = min(dim / 8, KP - 1);
      v_off[mt] = (4 * hh + trow) * (KP * 16) + ((slot ^ v_swz(trow)) << 4) + (dim & 7) * 2;
    } else {
      const int dim = min(mt * 32 + lq, KP * VEC - 1);
      v_off[mt] = 4 * hh * (KP * 16) + (((dim / 4) ^ v_swz(4 * hh)) << 4) + (dim & 3) * 4;
    }
  }

  f32x16 o[DM];
  float m = -INFINITY, l = 0.f;  // in log2 units: what the exponents subtract; this lane's part of the denominator
  f32x16 minus_m;                // PRE: what the scores' sums start from
#pragma unroll
  for (int r = 0; r < 16; ++r) minus_m[r] = 0.f;
#pragma unroll
  for (int mt = 0; mt < DM; ++mt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[mt][r] = 0.f;

  // (what the loop uses of earlier loads is waited for in front of it: there the requests must stay in flight)
  asm volatile("" : "+v"(ent));
  int now = next_key0();
  if (nstage > 0) issue(0, now);
#pragma unroll
  for (int j = 0; j < STEPS; ++j) asm volatile("" : "+v"(qf[j].v));
  for (int st = 0; st < nstage; ++st) {
    barrier_keep<0>();  // stage st has landed for everyone, and nobody still reads the other buffer
    const int next = next_key0();
    if (st + 1 < nstage) issue(st + 1, next);
    const unsigned char* const buf = smem + (st % NB) * S::STAGE;
    const int key0 = now + half * 32;
    if (busy && key0 < TK) {
      // (matrix phases go first where wavefronts compete: 609 -> 598 us at 33001 tokens, 64 of 516 blocks; with 128 channels, where there
      // are two wavefronts a SIMD, 43 -> 44 at 2 x 4096)
      if (kPrio) __builtin_amdgcn_s_setprio(1);
      f32x16 sc[KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[kt][r] = 0.f;
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
          const Vec16<T> kf = *reinterpret_cast<const Vec16<T>*>(buf + k_at + (half + kt) * 32 * (KP * 16) + (((2 * j + hh) ^ k_swz(lq)) << 4));
          if constexpr (BF) {
            sc[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf.v, qf[j].v, PRE && j == 0 ? minus_m : sc[kt], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) M::mma(kf.v[e], qf[j].v[e], sc[kt]);
          }
        }
      }
      if (kPrio) __builtin_amdgcn_s_setprio(0);
      // lane holds keys key0 + 32 kt + 8 (r / 4) + 4 hh + r % 4 of query lq
      if (now + 64 > TK) {
        int kb = key0 + 4 * hh;
        asm volatile("" : "+v"(kb));  // (left alone the compiler computes the indexes outside the branch)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (kb + kt * 32 + 8 * (r >> 2) + (r & 3) >= TK) sc[kt][r] = -INFINITY;
      }
      float mx = sc[0][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[kt][r]);
      // Any offset gives the same softmax while exp2 stays in range: it is raised, and what is summed up scaled, only when a score
      // passes it by kLazy. Each query decides for itself, whoever shares its wavefront.
      constexpr float kLazy = 8.f;
      const float mc = m == -INFINITY ? 0.f : m;
      mx = PRE ? mx + mc : mx * a.scale;
      if (__builtin_amdgcn_ballot_w64(mx > m + kLazy) != 0) {
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = mx > m + kLazy ? mx : m;
        const float alpha = m_new == m ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        const float by = m_new == -INFINITY ? 0.f : m_new - mc;
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int mt = 0; mt < DM; ++mt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[mt][r] *= alpha;
        if constexpr (PRE) {
#pragma unroll
          for (int r = 0; r < 16; ++r) minus_m[r] -= by;
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[kt][r] -= by;
        }
      }
      const float sub = m == -INFINITY ? 0.f : m;
      auto weight = [&](float x) { return __builtin_amdgcn_exp2f(PRE ? x : fmaf(x, a.scale, -sub)); };
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        if constexpr (BF) {
          bf16x8 pf[2];
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            bf16x2 p2, one2;
            p2[0] = static_cast<bf16_t>(weight(sc[kt][r]));
            p2[1] = static_cast<bf16_t>(weight(sc[kt][r + 1]));
            pf[r / 8][r % 8] = p2[0];
            pf[r / 8][r % 8 + 1] = p2[1];
            one2[0] = one2[1] = (bf16_t)1.f;
            // the denominator sums the probabilities as rounded: a key's share of numerator and denominator is then the same
#ifdef __HIP_DEVICE_COMPILE__
            l = __builtin_amdgcn_fdot2_f32_bf16(p2, one2, l, false);
#endif
          }
          if (kPrio) __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int mt = 0; mt < DM; ++mt) {
              bf16x8 vf = {};
#ifdef __HIP_DEVICE_COMPILE__
              typedef __attribute__((address_space(3))) s16x4* tr_ptr;
              const unsigned char* const p = buf + v_at + v_off[mt] + ((half + kt) * 32 + 16 * s) * (KP * 16);
              const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p));
              const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(p + 8 * (KP * 16)));
              const auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
              vf = __builtin_bit_cast(bf16x8, both);
#else
              (void)v_off;
#endif
              M::mma(vf, pf[s], o[mt]);
            }
          if (kPrio) __builtin_amdgcn_s_setprio(0);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float p = weight(sc[kt][r]);
            l += p;
#pragma unroll
            for (int mt = 0; mt < DM; ++mt) {
              const float vf = *reinterpret_cast<const float*>(buf + v_at + v_off[mt] + ((half + kt) * 32 + 8 * (r >> 2) + (r & 3)) * (KP * 16));
              M::mma(vf, p, o[mt]);
            }
          }
        }
      }
    }
    now = next;
  }

  // ---- wavefronts that shared queries: every second one hands its sums to the one before, which brings both to the larger of
  // their offsets and adds them; then the third to the first (a fixed order)
  if constexpr (KS > 1) {
#pragma unroll
    for (int step = 1; step < KS; step *= 2) {
      const bool gives = (wid & (2 * step - 1)) == step, takes = (wid & (2 * step - 1)) == 0;
      float* const box = reinterpret_cast<float*>(smem + (step == 1 ? wid >> 1 : 0) * S::HAND) + lane;
      __syncthreads();
      if (gives) {
        box[0] = m;
        box[64] = l;
#pragma unroll
        for (int mt = 0; mt < DM; ++mt)
#pragma unroll
          for (int r = 0; r < 16; ++r) box[(2 + mt * 16 + r) * 64] = o[mt][r];
      }
      __syncthreads();
      if (takes) {
        const float mo = box[0], top = fmaxf(m, mo);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top), fo = mo == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mo - top);
        m = top;
        l = l * f + box[64] * fo;
#pragma unroll
        for (int mt = 0; mt < DM; ++mt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[mt][r] = o[mt][r] * f + box[(2 + mt * 16 + r) * 64] * fo;
      }
    }
    if (wid % KS != 0) return;
  }

  // ---- lane holds O^T[dim = 32 mt + 8 (r / 4) + 4 hh + r % 4][query lq]
  l += __shfl_xor(l, 32, 64);
  if (qi >= rows) return;
  const int64_t pq = (int64_t)prob * a.Tq + row0 + qi;  // this query, counted over all
  const float inv = a.splits > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
  float* const po = a.part + (pq * a.splits + split) * D;
  T* const orow = out + b * a.os.batch + h * a.os.head + (int64_t)(row0 + qi) * a.os.token;
  if (a.splits > 1 && hh == 0) {
    float* const w = a.part + (int64_t)a.B * a.H * a.Tq * a.splits * D + (pq * a.splits + split) * 2;
    w[0] = m;
    w[1] = l;
  }
#pragma unroll
  for (int mt = 0; mt < DM; ++mt)
#pragma unroll
    for (int gr = 0; gr < 4; ++gr) {
      const int dim = mt * 32 + 8 * gr + 4 * hh;
      if (dim < D) {
        f32x4 ov;
#pragma unroll
        for (int e = 0; e < 4; ++e) ov[e] = o[mt][4 * gr + e] * inv;
        if (a.splits > 1) {
          *reinterpret_cast<f32x4*>(po + dim) = ov;
        } else if constexpr (BF) {
          bf16x4 ob;
#pragma unroll
          for (int e = 0; e < 4; ++e) ob[e] = static_cast<bf16_t>(ov[e]);
          *reinterpret_cast<bf16x4*>(orow + dim) = ob;
        } else {
          *reinterpret_cast<f32x4*>(orow + dim) = ov;
        }
      }
    }
}

// out = the splits' sums brought to one offset, added in a fixed order and divided; a thread four dims of a query
template <class T>
__global__ __launch_bounds__(256) void block_attn_join_kernel(BlockAttnArgs a, T* __restrict__ out, int D) {
  const int per = D / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = (int64_t)a.B * a.H * a.Tq;
  const int64_t pq = i / per;
  if (pq >= n) return;
  const int dim = (int)(i - pq * per) * 4, prob = (int)(pq / a.Tq), row = (int)(pq - (int64_t)prob * a.Tq), b = prob / a.H, h = prob - b * a.H;
  if (a.q_len && row >= a.q_len[b]) return;
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const f32x2* const ml = reinterpret_cast<const f32x2*>(a.part + n * a.splits * D) + pq * a.splits;
  const float* const po = a.part + pq * a.splits * D + dim;
  float top = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int AHEAD = 4;  // splits under way at a time
  for (int s0 = 0; s0 < a.splits; s0 += AHEAD) {
    f32x2 w[AHEAD];
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int s = min(s0 + u, a.splits - 1);
      w[u] = ml[s];
      v[u] = *reinterpret_cast<const f32x4*>(po + (int64_t)s * D);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (s0 + u >= a.splits) break;
      const float t = fmaxf(top, w[u][0]);
      const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - t), g = w[u][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w[u][0] - t);
      top = t;
      l = l * f + w[u][1] * g;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = acc[e] * f + v[u][e] * g;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* const orow = out + b * a.os.batch + (int64_t)row * a.os.token + h * a.os.head + dim;
#pragma unroll
  for (int e = 0; e < 4; ++e) orow[e] = from_f32<T>(acc[e] * inv);
}

struct AttnSplit { int ks, parts, splits; };
// How a call is shared out. Groups of up to 32, 64, 128 queries take 4, 2, 1 wavefronts a tile. Where that leaves compute units
// without work, bf16 groups are cut into parts of fewer tiles, whose keys more wavefronts share (16 heads of 64, 512 queries, 32 of 128
// blocks: 17.8 us, with the lists cut instead 16.7 + 4.5 for the join; floats, whose stages are twice as long, gain nothing), and then
// lists among several workgroups, as long as each of them keeps two stages (16 heads, one query, 32 blocks: 7.0 us with two, 8.8 with
// four, 17 uncut; 4 heads of floats, 300 queries, 20 blocks: 12.6, 16.6 and 53).
AttnSplit attn_split(const lc_sparse_args* a) {
  const int64_t groups = (int64_t)a->B * a->heads * lc_sparse_groups(a);
  const int rows = a->q_block < a->Tq ? a->q_block : a->Tq;
  AttnSplit r;
  r.ks = rows <= 32 ? 4 : rows <= 64 ? 2 : 1;
  if (a->dtype == LC_BF16)
    while (r.ks < 4 && groups * ((rows * r.ks + 127) / 128) < 512) r.ks *= 2;
  r.parts = (rows * r.ks + 127) / 128;
  const int64_t wgs = groups * r.parts, cpb = a->block / 64, most = ((int64_t)a->Tk + 63) / 64;
  const int64_t chunks = a->keep * cpb < most ? a->keep * cpb : most, stages = r.ks == 4 ? (chunks + 1) / 2 : chunks;
  const int64_t want = wgs < 256 ? (512 + wgs - 1) / wgs : 1, room = stages / 2, s = want < room ? want : room;
  r.splits = s < 1 ? 1 : (int)s;
  return r;
}

int check_attention(const lc_sparse_args* a) {
  int s = check_sparse_args(a);
  if (s != LC_OK) return s;
  const int64_t es = (int64_t)dtype_size(a->dtype), most = ((int64_t)1 << 30) / 64 / es;
  if (a->Tk > 1) {  // (the token stride of one key says nothing)
    if (a->k.token > most || a->v.token > most || a->k.token < 0 || a->v.token < 0) return op_fail(LC_ERR_SHAPE, "64 token strides of k and v must be within 2^30 bytes");
    if (a->k.token < a->head_dim || a->v.token < a->head_dim) return op_fail(LC_ERR_SHAPE, "the rows of k and of v must not overlap");
  }
  if (!strides_apart(a->out, a->B, a->Tq, a->heads)) return op_fail(LC_ERR_SHAPE, "the rows of out must not overlap");
  const int64_t groups = (int64_t)a->B * a->heads * lc_sparse_groups(a);
  if (groups > (int64_t)1 << 23) return op_fail(LC_ERR_SHAPE, "too many groups of queries");
  return LC_OK;
}

template <class T, int D, int KS, bool PRE> hipError_t run_block_attn(hipStream_t s, const BlockAttnArgs& a, const void* q, const void* k, const void* v, void* out) {
  constexpr int lds = BlockAttnShape<T, D, KS>::LDS;
  static_assert(lds <= 160 * 1024, "fits a compute unit");
  if (lds > 65536) {
    static std::atomic<uint64_t> done{0};  // a bit for each device
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(done.load() & bit)) {
      e = hipFuncSetAttribute((const void*)block_attn_kernel<T, D, KS, PRE>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
      done.fetch_or(bit);
    }
  }
  const unsigned grid = (unsigned)((int64_t)a.B * a.H * a.nq * a.parts * a.splits);
  block_attn_kernel<T, D, KS, PRE><<<grid, 256, lds, s>>>(a, (const T*)q, (const T*)k, (const T*)v, (T*)out);
  return hipGetLastError();
}
template <class T> hipError_t block_attn_dispatch(hipStream_t s, const BlockAttnArgs& a, int d, int ks, const void* q, const void* k, const void* v, void* out) {
#define LC_KS(D, PRE)                                                    \
  return ks == 1 ? run_block_attn<T, D, 1, PRE>(s, a, q, k, v, out)      \
         : ks == 2 ? run_block_attn<T, D, 2, PRE>(s, a, q, k, v, out)    \
                   : run_block_attn<T, D, 4, PRE>(s, a, q, k, v, out)
#define LC_GO(D)                                                         \
  case D:                                                                \
    if constexpr (sizeof(T) == 2 && D <= 64)                             \
      if (a.scale == 1.f) LC_KS(D, true);                                \
    LC_KS(D, false)
  switch (d) {
    LC_GO(8);
    LC_GO(16);
    LC_GO(32);
    LC_GO(40);
    LC_GO(64);
    LC_GO(128);
    default: return hipErrorInvalidValue;
  }
#undef LC_GO
#undef LC_KS
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" {

size_t lc_block_attention_workspace(const lc_sparse_args* a) {
  if (check_attention(a) != LC_OK) return 0;
  const int s = attn_split(a).splits;
  return s == 1 ? 0 : (size_t)a->B * a->heads * a->Tq * s * (a->head_dim + 2) * 4;
}

lc_status lc_op_block_attention(const lc_sparse_args* a, const void* q, const void* k, const void* v, const int32_t* index,
                                const int32_t* q_len, const int32_t* k_len, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  int s = check_attention(a);
  if (s == LC_OK) s = check_sparse_rows("q", q, a->q, a->dtype);
  if (s == LC_OK) s = check_sparse_rows("k", k, a->k, a->dtype);
  if (s == LC_OK) s = check_sparse_rows("v", v, a->v, a->dtype);
  if (s == LC_OK) s = check_sparse_rows("out", out, a->out, a->dtype);
  if (s != LC_OK) return (lc_status)s;
  if (!index) return (lc_status)op_fail(LC_ERR_ARG, "index is NULL");
  if (a->q_prescaled != 0 && a->q_prescaled != 1) return (lc_status)op_fail(LC_ERR_ARG, "q_prescaled must be 0 or 1");
  const size_t need = lc_block_attention_workspace(a);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return (lc_status)op_fail(LC_ERR_NOMEM, "workspace of %zu bytes is smaller than the %zu needed", workspace ? workspace_bytes : (size_t)0, need);
  if (need > 0 && (uintptr_t)workspace % 16) return (lc_status)op_fail(LC_ERR_ARG, "workspace must be 16-byte aligned");
  BlockAttnArgs k_;
  k_.qs = a->q; k_.ks = a->k; k_.vs = a->v; k_.os = a->out;
  if (a->Tk == 1) k_.ks.token = k_.vs.token = a->head_dim;  // (any stride says the same; this one puts rows that do not exist out of range)
  k_.index = index; k_.q_len = q_len; k_.k_len = k_len;
  k_.part = (float*)workspace;
  k_.scale = a->q_prescaled ? 1.f : attn_q_scale(a->head_dim);
  k_.B = a->B; k_.Tq = a->Tq; k_.Tk = a->Tk; k_.H = a->heads; k_.Hkv = a->kv_heads; k_.block = a->block; k_.q_block = a->q_block;
  k_.keep = a->keep; k_.nq = lc_sparse_groups(a);
  const AttnSplit sp = attn_split(a);
  k_.splits = sp.splits; k_.parts = sp.parts;
  const int64_t kvs = (int64_t)a->B * a->kv_heads;
  k_.unit = kvs % 8 == 0 ? a->heads / a->kv_heads : kvs * (a->heads / a->kv_heads) % 8 == 0 ? 1 : 0;
  const int64_t per = (int64_t)k_.nq * k_.parts * k_.splits;
  k_.per_prob = Div(per); k_.per_run = Div(per * (k_.unit > 0 ? k_.unit : 1));
  k_.by_splits = Div(k_.splits); k_.by_parts = Div(k_.parts); k_.by_H = Div(k_.H); k_.by_group = Div(k_.H / k_.Hkv);
  hipError_t e = a->dtype == LC_BF16 ? block_attn_dispatch<bf16_t>((hipStream_t)stream, k_, a->head_dim, sp.ks, q, k, v, out)
                                     : block_attn_dispatch<float>((hipStream_t)stream, k_, a->head_dim, sp.ks, q, k, v, out);
  if (e == hipSuccess && k_.splits > 1) {
    const int64_t n = (int64_t)a->B * a->heads * a->Tq * (a->head_dim / 4);
    const unsigned blocks = (unsigned)((n + 255) / 256);
    if (a->dtype == LC_BF16) block_attn_join_kernel<bf16_t><<<blocks, 256, 0, (hipStream_t)stream>>>(k_, (bf16_t*)out, a->head_dim);
    else block_attn_join_kernel<float><<<blocks, 256, 0, (hipStream_t)stream>>>(k_, (float*)out, a->head_dim);
    e = hipGetLastError();
  }
  return e == hipSuccess ? LC_OK : (lc_status)op_fail(LC_ERR_HIP, "block_attention: %s", hipGetErrorString(e));
}

}  // extern "C"
