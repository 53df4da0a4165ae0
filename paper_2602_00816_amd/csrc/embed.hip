// The token embedding at both points and the gradients of its tables.
//
// Row t of the output is s E[tok] (+ P[position]) with the scale s; in channel form the
// mean takes the tables' rows and the half difference eps times their directions' rows.
// The gradient entry of Hv for a table row is s / eps times the sum of the rows'
// half differences over the positions that hold its token.  Those positions are brought
// together by a stable sort of the tokens; every sum is then taken in fp64 in a fixed order.
#include <algorithm>

#include "kernels.h"

namespace fdh {

namespace {

constexpr int NT = 256;

// four floats of any element alignment (one 16-byte access)
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
__device__ inline float4 row4(const float* p, int64_t i) {
  const f4u v = *reinterpret_cast<const f4u*>(p + i);
  return make_float4(v.x, v.y, v.z, v.w);
}
__device__ inline void put4(float* p, int64_t i, float a, float b, float c, float d) {
  *reinterpret_cast<f4u*>(p + i) = f4u{a, b, c, d};
}
__device__ inline float4 row4(const bf16_t* p, int64_t i) {
  const uint2 u = *reinterpret_cast<const uint2*>(p + i);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xffff0000u));
}

// Forward: `lanes` threads per row (a power of two), four columns per thread and step, each
// output rounded once from fp64.  Bound by HBM: the tables' rows read, the pair written.  A
// token outside [0, V) has no row: its outputs are NaN, and bad_tok[0] (if given) is set.
template <typename T>
__global__ __launch_bounds__(NT) void embed_fwd_kernel(PairF x, int64_t ldx, const int32_t* tok, int64_t T_, int S, int dm, int V,
                                                       EmbedTables w, int lanes, int* bad_tok) {
  const int per = NT / lanes, l = threadIdx.x % lanes;
  for (int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / lanes; t < T_; t += (int64_t)gridDim.x * per) {
    const int tk = tok[t];
    const bool bad = tk < 0 || tk >= V;
    if (bad && bad_tok && l == 0) bad_tok[0] = 1;
    const T* e = (const T*)w.e + (bad ? 0 : (int64_t)tk * dm);
    const float* ve = w.ve ? w.ve + (bad ? 0 : (int64_t)tk * dm) : nullptr;
    const int64_t pr = w.p ? t % S * dm : 0;
    for (int c = 4 * l; c < dm; c += 4 * lanes) {
      const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
      const float4 a = row4(e, c), va = ve ? row4(ve, c) : none;
      const float4 b = w.p ? row4((const T*)w.p, pr + c) : none, vb = w.vp ? row4(w.vp, pr + c) : none;
      auto mean = [&](float p, float q) { return bad ? __builtin_nanf("") : (float)(w.scale * (double)p + (double)q); };
      auto half = [&](float p, float q) { return bad ? __builtin_nanf("") : (float)(w.eps * (w.scale * (double)p + (double)q)); };
      put4(x.m, t * ldx + c, mean(a.x, b.x), mean(a.y, b.y), mean(a.z, b.z), mean(a.w, b.w));
      put4(x.d, t * ldx + c, half(va.x, vb.x), half(va.y, vb.y), half(va.z, vb.z), half(va.w, vb.w));
    }
  }
}

// ---- stable sort of the tokens ---------------------------------------------------------
// Least significant digit first, 9 bits a pass, so one or two passes (V < 2^18).  A block
// takes a run of keys, each of its wavefronts a quarter of it.  A pass is two launches: the
// blocks' digit counts; then every block forms the places of its digits from the counts of
// all blocks and moves its keys there, 64 of a wavefront at a time in their order (the
// lanes of equal digit found by one ballot per bit).  The table's rows that no token has are
// zeros: blocks beyond the sort's write a part of the table in each launch, and so hide
// the sort, which is bound by latency; the rest is written beside the sums.
constexpr int BITS = 9, BINS = 1 << BITS, SORT_BLOCKS = 64, WAVES = NT / 64;

struct SortArgs {
  const int32_t* tok;                    // first pass: the keys (outside [0, V): V)
  const uint32_t *key, *pos;             // second pass
  uint32_t *okey, *opos;
  uint32_t* count;                       // [blocks][BINS]
  int64_t T, per;                        // keys per block, a multiple of NT
  int V, shift, blocks;
  float* zero;                           // table, or null
  int64_t zero4, zpart;                  // its float4s, and those that a launch sets (from zfrom on)
  int64_t zfrom;
};

__device__ inline uint32_t sort_key(const SortArgs& a, int64_t i) {
  if (!a.tok) return a.key[i];
  const int t = a.tok[i];
  return t < 0 || t >= a.V ? (uint32_t)a.V : (uint32_t)t;
}

__device__ inline void zero_part(const SortArgs& a, int block, int blocks) {
  const int64_t end = min(a.zfrom + a.zpart, a.zero4);
  for (int64_t i = a.zfrom + (int64_t)block * NT + threadIdx.x; i < end; i += (int64_t)blocks * NT)
    put4(a.zero, 4 * i, 0.f, 0.f, 0.f, 0.f);
}

__global__ __launch_bounds__(NT) void sort_count_kernel(SortArgs a) {
  const int b = blockIdx.x;
  if (b >= a.blocks) return zero_part(a, b - a.blocks, gridDim.x - a.blocks);
  __shared__ uint32_t h[BINS];
  for (int i = threadIdx.x; i < BINS; i += NT) h[i] = 0;
  __syncthreads();
  const int64_t end = min((b + 1) * a.per, a.T);
  for (int64_t i = b * a.per + threadIdx.x; i < end; i += NT) atomicAdd(&h[(sort_key(a, i) >> a.shift) & (BINS - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < BINS; i += NT) a.count[(int64_t)b * BINS + i] = h[i];
}

__global__ __launch_bounds__(NT) void sort_move_kernel(SortArgs a) {
  const int b = blockIdx.x;
  if (b >= a.blocks) return zero_part(a, b - a.blocks, gridDim.x - a.blocks);
  __shared__ uint32_t place[WAVES][BINS];   // counts, then the next place of every digit
  __shared__ uint32_t sum[WAVES];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i < WAVES * BINS; i += NT) (&place[0][0])[i] = 0;
  __syncthreads();
  const int64_t quarter = a.per / WAVES, from = b * a.per + w * quarter;
  const int64_t end = min(from + quarter, a.T);
  for (int64_t i = from + lane; i < end; i += 64) atomicAdd(&place[w][(sort_key(a, i) >> a.shift) & (BINS - 1)], 1u);
  // digits 2 tid and 2 tid + 1: their keys in all blocks and in the blocks before
  static_assert(BINS == 2 * NT, "two digits per thread");
  uint32_t all[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll 8
  for (int q = 0; q < a.blocks; ++q) {
    const uint2 c = *reinterpret_cast<const uint2*>(a.count + (int64_t)q * BINS + 2 * threadIdx.x);
    all[0] += c.x;
    all[1] += c.y;
    if (q < b) {
      before[0] += c.x;
      before[1] += c.y;
    }
  }
  uint32_t scan = all[0] + all[1];   // inclusive over the wavefront's lanes
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(scan, o, 64);
    if (lane >= o) scan += y;
  }
  if (lane == 63) sum[w] = scan;
  __syncthreads();   // (the wavefronts' counts too)
  uint32_t at = scan - all[0] - all[1];
  for (int q = 0; q < w; ++q) at += sum[q];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    uint32_t p = at + before[e];
#pragma unroll
    for (int q = 0; q < WAVES; ++q) {
      const uint32_t n = place[q][2 * threadIdx.x + e];
      place[q][2 * threadIdx.x + e] = p;
      p += n;
    }
    at += all[e];
  }
  __syncthreads();
  for (int64_t i0 = from; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool live = i < end;
    const uint32_t k = live ? sort_key(a, i) : 0u;
    const uint32_t dg = (k >> a.shift) & (BINS - 1);
    uint64_t same = __ballot(live);
#pragma unroll
    for (int j = 0; j < BITS; ++j) {
      const uint64_t m = __ballot((dg >> j) & 1);
      same &= (dg >> j) & 1 ? m : ~m;
    }
    const uint32_t ahead = (uint32_t)__popcll(same & (((uint64_t)1 << lane) - 1));
    const uint32_t to = live ? place[w][dg] + ahead : 0u;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();   // every lane has read its place
    if (live && ahead == 0) place[w][dg] = to + (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live) {
      a.okey[to] = k;
      a.opos[to] = a.tok ? (uint32_t)i : a.pos[i];
    }
  }
}

// Position rows: the sum over the batch's rows, 16 of them in flight; rows S .. are set to zero.
struct PosArgs {
  float* hv;       // null: no positions
  const float* dx;
  int64_t ld;
  int B, S, dm, acc;
  double inv_eps;
  int64_t n4;      // float4s of the table's rows
};
__device__ inline void pos_part(const PosArgs& a, int block, int blocks) {
  const int n4 = a.dm / 4;
  for (int64_t i = (int64_t)block * NT + threadIdx.x; i < a.n4; i += (int64_t)blocks * NT) {
    const int64_t r = i / n4;
    const int c = 4 * (int)(i - r * n4);
    if (r >= a.S) {
      put4(a.hv, 4 * i, 0.f, 0.f, 0.f, 0.f);
      continue;
    }
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    constexpr int U = 16;
    for (int b0 = 0; b0 < a.B; b0 += U) {
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = row4(a.dx, ((int64_t)min(b0 + u, a.B - 1) * a.S + r) * a.ld + c);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (b0 + u < a.B) { s[0] += (double)x[u].x; s[1] += (double)x[u].y; s[2] += (double)x[u].z; s[3] += (double)x[u].w; }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] *= a.inv_eps;
    if (a.acc) {
      const float4 h = row4(a.hv, 4 * i);
      s[0] += h.x; s[1] += h.y; s[2] += h.z; s[3] += h.w;
    }
    put4(a.hv, 4 * i, (float)s[0], (float)s[1], (float)s[2], (float)s[3]);
  }
}

// ---- sums of the sorted rows -----------------------------------------------------------
// A wavefront takes R consecutive sorted rows at 256 columns (four a lane), 16 rows in flight.
// A token whose rows all lie in the chunk gets its sum at once.  One whose rows go beyond
// it leaves fp64 parts, [chunk][2][dm]: in 0 the sum of the chunk's first token when the
// chunk before holds that token too, in 1 that of its last token when it begins here and
// goes on.  embed_join_kernel adds the parts of such a token from the chunk in which it
// begins.  However often a token occurs, no wavefront adds more than R rows and the join's
// wavefronts a quarter of R-th as many parts, one after the other: where one token is everywhere that
// is most of the time (8192 tokens of 32000 x 2048: 83 us spread evenly, 108 with half of them
// one token, 132 with all).
struct SumArgs {
  const uint32_t *key, *pos;
  const float* dx;
  int64_t ld, T;
  int dm, V;
  float* hv;
  double mul;      // scale / eps
  int acc;
  double* part;
  int64_t chunks;  // chunks of R rows
  int64_t blocks;  // workgroups that add; then pblocks that add positions (the same rows again, from the
  int pblocks;     // caches), then those that set rows zfrom .. V - 1 that no token has to zero
  int zfrom;
  PosArgs posn;
};

// ZROWS rows per wavefront: whether a token has them is looked up in the sorted keys (a lane each)
constexpr int ZROWS = 8;
__device__ inline void zero_rows(const SumArgs& a, int64_t block) {
  const int lane = threadIdx.x & 63;
  const int64_t r0 = a.zfrom + (block * WAVES + (threadIdx.x >> 6)) * ZROWS;
  const uint32_t r = (uint32_t)min(r0 + lane % ZROWS, (int64_t)a.V - 1);
  int64_t lo = 0, hi = a.T;   // first sorted position of a key >= r
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (a.key[mid] < r) lo = mid + 1;
    else hi = mid;
  }
  const uint64_t there = __ballot(lo < a.T && a.key[min(lo, a.T - 1)] == r);
  for (int i = 0; i < ZROWS; ++i) {
    if (r0 + i >= a.V || (there >> i & 1)) continue;
    for (int c = 4 * lane; c < a.dm; c += 256) put4(a.hv, (r0 + i) * a.dm + c, 0.f, 0.f, 0.f, 0.f);
  }
}

__device__ inline void put_sum(const SumArgs& a, uint32_t tk, int c, const double (&s)[4]) {
  const int64_t o = (int64_t)tk * a.dm + c;
  double x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = s[e] * a.mul;
  if (a.acc) {
    const float4 h = row4(a.hv, o);
    x[0] += h.x; x[1] += h.y; x[2] += h.z; x[3] += h.w;
  }
  put4(a.hv, o, (float)x[0], (float)x[1], (float)x[2], (float)x[3]);
}

template <int R>
__global__ __launch_bounds__(NT) void embed_sum_kernel(SumArgs a) {
  static_assert(R <= 64, "a lane for every row of a chunk");
  constexpr int U = 16;
  if (blockIdx.x >= a.blocks) {
    const int64_t b = blockIdx.x - a.blocks;
    if (b < a.pblocks) pos_part(a.posn, (int)b, a.pblocks);
    else zero_rows(a, b - a.pblocks);
    return;
  }
  const int64_t chunk = blockIdx.x % a.chunks, s0 = chunk * R;
  const int n = (int)min((int64_t)R, a.T - s0);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = ((int)(blockIdx.x / a.chunks) * WAVES + wave) * 256;
  if (c0 >= a.dm) return;
  const int c = c0 + 4 * lane;
  const bool on = c < a.dm;
  const int col = on ? c : 0;
  const int64_t mine = s0 + min(lane, n - 1);
  const uint32_t kk = a.key[mine], pp = a.pos[mine];
  const uint32_t none = 0xFFFFFFFFu;
  const uint32_t prev = s0 > 0 ? a.key[s0 - 1] : none;
  const uint32_t next = s0 + n < a.T ? a.key[s0 + n] : none;
  auto key_at = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)kk, i); };
  bool begins = key_at(0) != (uint32_t)__builtin_amdgcn_readfirstlane((int)prev);
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i0 = 0; i0 < n; i0 += U) {
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)pp, min(i0 + u, n - 1));
      x[u] = row4(a.dx, (int64_t)p * a.ld + col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u;
      if (i >= n) break;
      s[0] += (double)x[u].x; s[1] += (double)x[u].y; s[2] += (double)x[u].z; s[3] += (double)x[u].w;
      const bool last = i == n - 1;
      const uint32_t tk = key_at(i);
      const uint32_t after = last ? (uint32_t)__builtin_amdgcn_readfirstlane((int)next) : key_at(i + 1);
      if (!last && after == tk) continue;
      if (tk < (uint32_t)a.V && on) {
        if (begins && after != tk) {
          put_sum(a, tk, c, s);
        } else {
          double* o = a.part + (2 * chunk + (begins ? 1 : 0)) * a.dm + c;
          *reinterpret_cast<double2*>(o) = make_double2(s[0], s[1]);
          *reinterpret_cast<double2*>(o + 2) = make_double2(s[2], s[3]);
        }
      }
      begins = true;
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = 0.0;
    }
  }
}

// One workgroup per chunk and 256 columns; those of chunks in which no token begins that
// goes on have nothing to do.  The wavefronts add a quarter of the parts each.
template <int R>
__global__ __launch_bounds__(NT) void embed_join_kernel(SumArgs a) {
  __shared__ double sh[WAVES][256];
  const int64_t chunk = blockIdx.x, s0 = chunk * R, s1 = s0 + R;
  if (s1 >= a.T) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (all keys at once: each wait is some 1.5 us of the kernel's 5)
  const uint32_t before = a.key[s0 > 0 ? s0 - 1 : 0], head = a.key[s0], tk = a.key[s1 - 1];
  auto at = [&](int64_t m) { return a.key[min((chunk + 1 + m + lane) * R, a.T - 1)]; };
  uint32_t after = at(0);
  if ((uint32_t)__builtin_amdgcn_readfirstlane((int)after) != tk || tk >= (uint32_t)a.V) return;
  if (s0 > 0 && head == tk && before == tk) return;   // it began before
  // chunks after this one whose first row is of this token
  int64_t m = 0;
  for (;;) {
    const uint64_t hit = __ballot((chunk + 1 + m + lane) * R < a.T && after == tk);
    const int k = ~hit ? __ffsll((unsigned long long)~hit) - 1 : 64;
    m += k;
    if (k < 64) break;
    after = at(m);
  }
  const int c = (int)blockIdx.y * 256 + 4 * lane;
  const bool on = c < a.dm;
  const int col = on ? c : 0;
  const int64_t per = (m + WAVES - 1) / WAVES, lo = wave * per, hi = min(lo + per, m);
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  const double* base = a.part + 2 * (chunk + 1) * a.dm + col;
  const double2 own0 = *reinterpret_cast<const double2*>(base - a.dm), own1 = *reinterpret_cast<const double2*>(base - a.dm + 2);
  constexpr int U = 16;
  for (int64_t q = lo; q < hi; q += U) {
    double2 x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const double* p = base + 2 * min(q + u, hi - 1) * a.dm;
      x[u] = *reinterpret_cast<const double2*>(p);
      y[u] = *reinterpret_cast<const double2*>(p + 2);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (q + u < hi) { s[0] += x[u].x; s[1] += x[u].y; s[2] += y[u].x; s[3] += y[u].y; }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sh[wave][4 * lane + e] = s[e];
  __syncthreads();
  if (wave != 0 || !on) return;
  const double own[4] = {own0.x, own0.y, own1.x, own1.y};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s[e] = own[e];
#pragma unroll
    for (int q = 0; q < WAVES; ++q) s[e] += sh[q][4 * lane + e];
  }
  put_sum(a, tk, c, s);
}

// ---- a few tokens: one launch, no sort -----------------------------------------------------
// A workgroup per position and 1024 columns: the first position of a token adds the rows of all of
// them in their order (eight in flight), the others have nothing to do.  The rows that no token has
// and the positions come behind, as above.  2 tokens, 11784 x 112: 23 -> 7 us.
constexpr int FEW = 256;
static_assert(FEW == NT, "a thread for every position");
__global__ __launch_bounds__(NT) void embed_few_kernel(SumArgs a, const int32_t* tok) {
  const int T_ = (int)a.T, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (blockIdx.x >= a.blocks) {
    const int64_t b = blockIdx.x - a.blocks;
    if (b < a.pblocks) return pos_part(a.posn, (int)b, a.pblocks);
    const int64_t r0 = ((b - a.pblocks) * WAVES + w) * ZROWS;
    int own[FEW / 64];
#pragma unroll
    for (int k = 0; k < FEW / 64; ++k) own[k] = tok[min(lane + 64 * k, T_ - 1)];
    for (int i = 0; i < ZROWS && r0 + i < a.V; ++i) {
      bool hit = false;
#pragma unroll
      for (int k = 0; k < FEW / 64; ++k) hit |= own[k] == (int)(r0 + i);
      if (__ballot(hit)) continue;
      for (int c = 4 * lane; c < a.dm; c += 256) put4(a.hv, (r0 + i) * a.dm + c, 0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  __shared__ uint64_t same[FEW / 64];
  const int t = (int)(blockIdx.x % a.chunks), c = 4 * ((int)(blockIdx.x / a.chunks) * NT + (int)threadIdx.x);
  const int tk = tok[t];
  const uint64_t m = __ballot((int)threadIdx.x < T_ && tok[min((int)threadIdx.x, T_ - 1)] == tk);
  if (lane == 0) same[w] = m;
  __syncthreads();
  uint64_t left[FEW / 64];
#pragma unroll
  for (int k = 0; k < FEW / 64; ++k) left[k] = same[k];
  auto next = [&]() {   // the lowest position left, or -1
    int p = -1;
#pragma unroll
    for (int k = FEW / 64 - 1; k >= 0; --k)
      if (left[k]) p = 64 * k + __ffsll((unsigned long long)left[k]) - 1;
#pragma unroll
    for (int k = 0; k < FEW / 64; ++k)
      if (p >> 6 == k) left[k] &= left[k] - 1;
    return p;
  };
  int p = next();
  if (p != t || tk < 0 || tk >= a.V || c >= a.dm) return;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  constexpr int U = 8;
  while (p >= 0) {
    float4 x[U];
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p < 0) continue;
      x[u] = row4(a.dx, (int64_t)p * a.ld + c);
      n = u + 1;
      p = next();
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < n) { s[0] += (double)x[u].x; s[1] += (double)x[u].y; s[2] += (double)x[u].z; s[3] += (double)x[u].w; }
  }
  put_sum(a, (uint32_t)tk, c, s);
}

// rows per chunk of the sums
int chunk_rows(int64_t T_) { return T_ <= 16384 ? 32 : 64; }

struct EmbedScratch {   // carve of the backward's scratch (bytes)
  size_t key[2], pos[2], count, part, total;
};
EmbedScratch embed_carve(int64_t T_, int dm) {
  EmbedScratch s;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  for (int q = 0; q < 2; ++q) {
    s.key[q] = take((size_t)T_ * 4);
    s.pos[q] = take((size_t)T_ * 4);
  }
  s.count = take((size_t)SORT_BLOCKS * BINS * 4);
  const size_t chunks = ((size_t)T_ + 31) / 32;   // (of 32 rows: as many or more than are used)
  s.part = take(chunks * 2 * dm * 8);
  s.total = T_ > FEW ? at : 0;
  return s;
}

}  // namespace

template <typename T>
hipError_t launch_embed_fwd(PairF x, int64_t ldx, const int32_t* tok, int64_t T_, int S, int dm, int V, const EmbedTables& w,
                            int* bad_tok, hipStream_t s) {
  if (T_ == 0) return hipSuccess;
  int lanes = 2;
  while (lanes < NT && 4 * lanes < dm) lanes *= 2;
  // (a launch ends at 2^32 threads)
  const dim3 grid((unsigned)std::min<int64_t>(1 << 22, ceil_div(T_, NT / lanes)));
  hipLaunchKernelGGL((embed_fwd_kernel<T>), grid, dim3(NT), 0, s, x, ldx, tok, T_, S, dm, V, w, lanes, bad_tok);
  return hipGetLastError();
}
template hipError_t launch_embed_fwd<float>(PairF, int64_t, const int32_t*, int64_t, int, int, int, const EmbedTables&, int*, hipStream_t);
template hipError_t launch_embed_fwd<bf16_t>(PairF, int64_t, const int32_t*, int64_t, int, int, int, const EmbedTables&, int*, hipStream_t);

size_t embed_scratch_bytes(int64_t T_, int dm) { return embed_carve(T_, dm).total; }

hipError_t launch_embed_bwd(const EmbedGrad& o, const int32_t* tok, const float* dxd, int64_t ld, int B, int S, int dm, int V,
                            void* scratch, hipStream_t s) {
  const int64_t T_ = (int64_t)B * S;
  const bool acc = o.acc;
  const int64_t zero4 = acc ? 0 : (int64_t)V * dm / 4;
  if (T_ == 0) {
    const hipError_t r = acc ? hipSuccess : launch_fill_f32(o.e, (int64_t)V * dm, 0.f, s);
    return r != hipSuccess || !o.p || o.acc_p ? r : launch_fill_f32(o.p, o.rows * dm, 0.f, s);
  }
  SumArgs u{};
  u.dx = dxd;
  u.ld = ld;
  u.T = T_;
  u.dm = dm;
  u.V = V;
  u.hv = o.e;
  u.mul = o.mul;
  u.acc = acc;
  const int64_t pos4 = o.p ? (o.acc_p ? std::min<int64_t>(o.rows, S) : o.rows) * (dm / 4) : 0;
  u.posn = PosArgs{o.p, dxd, ld, B, S, dm, o.acc_p, o.inv_eps, pos4};
  u.pblocks = (int)std::min<int64_t>(65536, ceil_div(pos4, NT));
  if (T_ <= FEW) {
    u.chunks = T_;
    u.blocks = T_ * ceil_div(dm, 4 * NT);
    const dim3 grid((unsigned)(u.blocks + u.pblocks + (acc ? 0 : ceil_div(V, ZROWS * WAVES))));
    hipLaunchKernelGGL(embed_few_kernel, grid, dim3(NT), 0, s, u, tok);
    return hipGetLastError();
  }
  char* ws = (char*)scratch;
  const EmbedScratch sc = embed_carve(T_, dm);
  SortArgs a{};
  a.T = T_;
  a.V = V;
  a.blocks = (int)std::min<int64_t>(SORT_BLOCKS, ceil_div(T_, 512));
  a.per = (int64_t)ceil_div(T_, (int64_t)a.blocks * NT) * NT;
  a.blocks = (int)ceil_div(T_, a.per);
  a.count = (uint32_t*)(ws + sc.count);
  a.zero = o.e;
  a.zero4 = zero4;
  const int passes = V + 1 > BINS ? 2 : 1;
  // an eighth of the table in each launch, in whole rows (8192 tokens, 32000 x 2048: about as long as
  // the sort takes)
  const int64_t zrows = zero4 ? V / 8 : 0;
  a.zpart = zrows * (dm / 4);
  const int zblocks = (int)std::min<int64_t>(512, ceil_div(a.zpart, NT));
  for (int p = 0; p < 2 * passes; ++p) {
    a.tok = p < 2 ? tok : nullptr;
    a.key = (const uint32_t*)(ws + sc.key[0]);
    a.pos = (const uint32_t*)(ws + sc.pos[0]);
    a.okey = (uint32_t*)(ws + sc.key[p / 2]);
    a.opos = (uint32_t*)(ws + sc.pos[p / 2]);
    a.shift = p / 2 * BITS;
    a.zfrom = p * a.zpart;
    if (p % 2 == 0) hipLaunchKernelGGL(sort_count_kernel, dim3(a.blocks + zblocks), dim3(NT), 0, s, a);
    else hipLaunchKernelGGL(sort_move_kernel, dim3(a.blocks + zblocks), dim3(NT), 0, s, a);
  }
  u.key = a.okey;
  u.pos = a.opos;
  u.part = (double*)(ws + sc.part);
  const int R = chunk_rows(T_);
  const unsigned chunks = ceil_div(T_, R), cols = ceil_div(dm, 256);
  u.chunks = chunks;
  u.blocks = (int64_t)chunks * ceil_div(cols, WAVES);
  u.zfrom = (int)(2 * passes * zrows);
  const dim3 gs((unsigned)(u.blocks + u.pblocks + (zero4 ? ceil_div(V - u.zfrom, ZROWS * WAVES) : 0))), gj(chunks, cols);
  if (R == 32) {
    hipLaunchKernelGGL(embed_sum_kernel<32>, gs, dim3(NT), 0, s, u);
    if (chunks > 1) hipLaunchKernelGGL(embed_join_kernel<32>, gj, dim3(NT), 0, s, u);
  } else {
    hipLaunchKernelGGL(embed_sum_kernel<64>, gs, dim3(NT), 0, s, u);
    hipLaunchKernelGGL(embed_join_kernel<64>, gj, dim3(NT), 0, s, u);
  }
  return hipGetLastError();
}

}  // namespace fdh
