// Attention with masks, capped scores and a distance bias for gfx950 (MI355X).  The tile code is that of the unmasked kernels
// (attn_device.h): 32 query rows a wavefront, S^T = K Q^T and O^T += V^T P^T on the 32x32x16 bf16 MFMA, 64 keys a tile.
//
//   s = scale <q, k>;  with a cap  C tanh(s / C);  with slopes  s - slope_h |pos - j|,  pos = row + keys - rows of the sequence
//   key j is seen by a row  iff  (not causal or j <= pos or j < prefix) and (no ids or the ids agree and are not negative)
//   O = sum over seen keys exp(s - lse) v,  lse = ln sum exp(s);  a row that sees nothing gets 0 and -inf.
//
// A row's causal and prefix mask is one bound: keys under max(pos + 1, prefix).  Tiles that no row of an item sees are not
// loaded (for document ids a small kernel takes the range of every tile first); tiles that every row sees wholly are not
// masked; in the others a dead score becomes -inf, one interval test per score plus one comparison of ids.
//
// What a row does not see may hold anything.  Scores are replaced, not added to, so a NaN key has no effect; a probability of
// 0 times a NaN or infinite value would be NaN, so the values of a masked tile are made finite in LDS (each wavefront looks at
// the rows that it loaded itself), and an item one of whose rows does see such a value adds it behind the loop.
//
// Two sums of a row: of the probabilities as rounded for the second contraction, which O is divided by (a convex combination
// of values whatever the rounding did), and of the fp32 ones, which the log-sum-exp is taken of.
#include "attn_device.h"
#include "masked_attn.h"

namespace dit {

constexpr float kLn2 = 0.69314718055994530942f;
[[maybe_unused]] constexpr float kNoReference = -3.0e38f;  // of a row that has seen no key

// The last of the first n sequences whose FIRST is not behind idx.
template <uint32_t MaskedSeq::*FIRST>
__device__ __forceinline__ const MaskedSeq& find_seq(const MaskedParams& p, int n, uint32_t idx) {
  int j = 0;
  if (n > 1) {
    static_assert(kMaskedSeqs == 64, "a lane for each sequence");
    const int lane = threadIdx.x & 63, i = lane < n ? lane : 0;
    j = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(lane < n && p.seq[i].*FIRST <= idx));
  }
  return p.seq[__builtin_amdgcn_readfirstlane(j)];
}

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const int y = __shfl_xor(x, d);
    x = y < x ? y : x;
  }
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x) { return ~wave_min(~x); }

// Ids of n consecutive places from ids, one a lane (n at most 64 counts).
__device__ __forceinline__ DocTile doc_range(const int32_t* ids, int n) {
  const int lane = threadIdx.x & 63;
  const int id = ids[lane < n ? lane : 0], one = __builtin_amdgcn_readfirstlane(id);
  DocTile r = {one, one, one, 0};
  if (one < 0 || __builtin_amdgcn_ballot_w64(id != one) != 0) {  // not all of one document
    r.any_lo = wave_min(id);
    r.lo = wave_min(id < 0 ? INT32_MAX : id);
    r.hi = wave_max(id < 0 ? -1 : id);
  }
  return r;
}

// Id ranges of all key tiles of a launch, a wavefront each: 4 us with its launch, which spares the attention kernel the tiles of
// other documents (two thirds of 6 x 4352 rows in three documents).
__global__ void __launch_bounds__(256) masked_doc_tiles_kernel(MaskedParams p, uint32_t n_tiles) {
  const uint32_t tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= n_tiles) return;
  const MaskedSeq& s = find_seq<&MaskedSeq::tile0>(p, p.n, tile);
  const int key0 = (int)(tile - s.tile0) * 64;
  const DocTile r = doc_range(p.k_doc + s.kv_start + key0, s.kv_len - key0);
  if ((threadIdx.x & 63) == 0) p.doc_tiles[tile] = r;
}

// The tiles [.., end) of a part that any row of an item sees, in order: 64 at a time from their id ranges, or simply all.
struct LiveTiles {
  const DocTile* ranges;  // of the sequence, or nullptr
  DocTile mine;           // ids of the item's rows
  int end, base;
  uint64_t live, pure;    // of base .. base + 63; pure: all rows and keys have the same document

  __device__ __forceinline__ void look(int t) {
    base = t;
    const int i = t + (int)(threadIdx.x & 63);
    const DocTile r = ranges[i < end ? i : end - 1];
    live = __builtin_amdgcn_ballot_w64(i < end && r.lo <= mine.hi && r.hi >= mine.lo);
    pure = __builtin_amdgcn_ballot_w64(r.any_lo == r.hi && mine.any_lo == r.hi && mine.hi == r.hi);
  }
  // The first live tile from t on, or end.
  __device__ __forceinline__ int next(int t) {
    if (ranges == nullptr) return t < end ? t : end;
    while (t < end) {
      if (t >= base + 64) look(t);
      const uint64_t rest = live >> (t - base);
      if (rest != 0) return t + __builtin_ctzll(rest);
      t = base + 64;
    }
    return end;
  }
  __device__ __forceinline__ bool is_pure(int t) const { return ranges == nullptr || ((pure >> (t - base)) & 1) != 0; }
};

// Scores of a lane: element i of block kb is key 32 kb + 8 (i / 4) + (i % 4) + 4 hh of the tile.
__device__ __forceinline__ constexpr int key_of(int kb, int i) { return 32 * kb + 8 * (i >> 2) + (i & 3); }

// C tanh(s / C) log2(e) of a raw score, as a polynomial where it is small and 1 - 2 / (exp(2 y) + 1) of y = s / C, whose limits
// need no clamp, where that keeps its relative precision: either is within 1e-6 of the score, most of it the roundings of 2 y, the
// exponential and the reciprocal next to a quarter of C (the polynomial is off by 4e-7).
__device__ __forceinline__ float small_cap(const MaskedParams& p, float x) {
  const float z = x * x;
  return x * __builtin_fmaf(z, __builtin_fmaf(z, p.poly[2], p.poly[1]), p.poly[0]);
}
__device__ __forceinline__ float capped(const MaskedParams& p, float x) {
  const float e = __builtin_amdgcn_exp2f(x * p.tanh_in);
  const float large = __builtin_fmaf(-2.f * p.cap_log2, __builtin_amdgcn_rcpf(e + 1.f), p.cap_log2);
  return __builtin_fabsf(x) <= p.poly_up_to ? small_cap(p, x) : large;
}

// Raw scores -> scores whose product with the kernel's c is the base-2 exponent (c is 1 with a cap, else |scale| log2 e).
// at: pos - first key of the tile - 4 hh of this lane;  slope: slope log2(e) / c.
// small (the same in the whole wavefront): no score exceeds p.small in absolute value, and the cap is the polynomial alone: four
// instructions a score instead of nine and an exponential and a reciprocal, which take four times as long each.
template <int NKB, bool CAP, bool BIAS>
__device__ __forceinline__ void shape_scores(f32x16 (&s)[NKB], const MaskedParams& p, bool small, float slope, int at) {
  if constexpr (CAP) {
    if (small) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = small_cap(p, s[kb][i]);
    } else {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = capped(p, s[kb][i]);
    }
  }
  if constexpr (BIAS) {
    const float base = (float)at;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = __builtin_fmaf(-slope, __builtin_fabsf(base - (float)key_of(kb, i)), s[kb][i]);
  }
}

// What a lane's row sees of a tile: keys lo <= key < hi of it, less 4 hh, whose ids are `doc` if there are ids.
struct LaneMask {
  int lo;
  unsigned n;
  __device__ __forceinline__ bool dead(int kb, int i) const { return (unsigned)(key_of(kb, i) - lo) >= n; }
};

typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
typedef __attribute__((address_space(3))) i32x4 lds_i32x4;
typedef __attribute__((address_space(3))) uint32_t lds_u32;

// Dead scores := -inf.  docs: LDS byte of the tile's ids, hh as everywhere.
template <int NKB>
__device__ __forceinline__ void mask_scores(f32x16 (&s)[NKB], LaneMask m, bool have_docs, uint32_t docs, int doc, int hh) {
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[kb][i] = m.dead(kb, i) ? -__builtin_inff() : s[kb][i];
  if (have_docs)
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const i32x4 id = *(lds_i32x4*)(uintptr_t)(docs + (uint32_t)(32 * kb + 8 * g + 4 * hh) * 4u);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[kb][4 * g + j] = id[j] != doc ? -__builtin_inff() : s[kb][4 * g + j];
      }
}

// A mask of 64 keys from its words, which readfirstlane returns as signed numbers: key 31 is not the sign of the others.
__host__ __device__ constexpr uint64_t mask_of_words(int lo, int hi) { return (uint64_t)(uint32_t)lo | (uint64_t)(uint32_t)hi << 32; }
static_assert(mask_of_words(INT32_MIN, 0) == 1ull << 31 && mask_of_words(-1, INT32_MIN) == 0x80000000FFFFFFFFull, "no sign extension");

// Whether this lane's row sees one of the keys whose bits are set.
template <int NKB>
__device__ __forceinline__ bool sees(const f32x16 (&s)[NKB], uint64_t keys, int hh) {
  bool any = false;
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) any |= s[kb][i] != -__builtin_inff() && ((keys >> (key_of(kb, i) + 4 * hh)) & 1) != 0;
  return any;
}

// Whether either lane of a row says so: they hold the scores of different keys, and other elements of the result.
__device__ __forceinline__ bool either_half(bool x) { return x | (__shfl_xor((int)x, 32) != 0); }

// Which half of its wavefront a lane is in; recomputed where it is needed.
__device__ __forceinline__ int half_of(int tid) {
  asm volatile("" : "+v"(tid));
  return (tid >> 5) & 1;
}

// State of a lane's row.
struct RowState {
  float m_ref;  // reference of the exponent, see tile_softmax
  float l;      // sum of the rounded probabilities (this half-wave's keys)
  float lx;     // sum of the fp32 ones
};

// Online softmax of one tile, as tile_softmax in attn_device.h, with the fp32 sum and for rows that may have seen nothing yet.
template <int NKB, int NDB, bool LSE>
__device__ __forceinline__ void masked_softmax(f32x16 (&s)[NKB], float mx, float c, uint32_t (&pb)[NKB][8], f32x16 (&o)[NDB], RowState& r) {
  const bool grow = (mx - r.m_ref) * c > kRescaleLog2;
  if (__builtin_amdgcn_ballot_w64(grow) != 0) {
    const float m_new = grow ? mx : r.m_ref;
    const float alpha = __builtin_amdgcn_exp2f((r.m_ref - m_new) * c);
    r.m_ref = m_new;
    r.l *= alpha;
    if constexpr (LSE) r.lx *= alpha;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
  }
  const float mc = __builtin_fmaxf(r.m_ref * c, -3.0e38f);  // finite, so that a dead score gives 0 in a row without a reference
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
#pragma unroll
      for (int i = 8 * g; i < 8 * g + 8; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], c, -mc));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i + 1], c, -mc));
        if constexpr (LSE) r.lx += p0 + p1;
        pb[kb][i >> 1] = pack_bf16x2(p0, p1);
      }
      SCHED_FENCE();
    }
  // Finished here, as in tile_softmax.
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
    asm volatile("" : "+v"(pb[kb][0]), "+v"(pb[kb][1]), "+v"(pb[kb][2]), "+v"(pb[kb][3]), "+v"(pb[kb][4]), "+v"(pb[kb][5]),
                      "+v"(pb[kb][6]), "+v"(pb[kb][7]));
}

__device__ __forceinline__ bool pair_not_finite(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// Values that are not finite of V rows in LDS become 0: N chunks of 16 bytes a lane, `step` apart from `addr`.  Returns the mask
// of the chunks that held one.
template <int N>
__device__ __forceinline__ uint32_t make_finite(uint32_t addr, uint32_t step) {
  uint32_t found = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    lds_u32x4* at = (lds_u32x4*)(uintptr_t)(addr + i * step);
    u32x4 w = *at;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) bad |= pair_not_finite(w[k]);
    if (bad) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((w[k] & 0x7F80u) == 0x7F80u) w[k] &= 0xFFFF0000u;
        if ((w[k] & 0x7F800000u) == 0x7F800000u) w[k] &= 0xFFFFu;
      }
      *at = w;
      found |= 1u << i;
    }
  }
  return found;
}

// Behind the loop of an item some of whose rows (poison: this lane's row, in both of its lanes) see a value that is not finite in
// a masked tile: such values of keys [key0, key1), key stride `step` in blocks of `run`, are added to the rows that see them, until
// nothing can change any more.  Slow, and seldom: about a microsecond a key.
template <class T>
__device__ __forceinline__ void add_not_finite(const MaskedParams& p, const char* vbase, const int32_t* kdoc, int key0, int key1, int run,
                                               int step, int klim, int doc, int hh, bool poison, f32x16 (&o)[T::NDB]) {
  for (int b = key0; b < key1; b += step)
    for (int j = b; j < b + run && j < key1; ++j) {
      const uint32_t* row = reinterpret_cast<const uint32_t*>(vbase + (int64_t)j * p.v_stride_b);
      const uint32_t w = row[threadIdx.x & (T::D / 2 - 1)];  // a pair of elements in each of the first D / 2 lanes
      const uint64_t pairs = __builtin_amdgcn_ballot_w64(pair_not_finite(w));
      if (pairs == 0) continue;
      const bool seen = j < klim && (kdoc == nullptr || kdoc[j] == doc);
      bool all_nan = true;
#pragma unroll
      for (int db = 0; db < T::NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int d = 32 * db + 8 * (i >> 2) + (i & 3);  // and 4 more in the upper half of the wavefront
          const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)w, d >> 1), hi = (uint32_t)__builtin_amdgcn_readlane((int)w, (d >> 1) + 2);
          const uint32_t x = hh ? hi : lo, bits = d & 1 ? x & 0xFFFF0000u : x << 16;
          const float sum = o[db][i] + __builtin_bit_cast(float, bits);
          o[db][i] = seen && (bits & 0x7F800000u) == 0x7F800000u ? sum : o[db][i];
          all_nan &= o[db][i] != o[db][i];
          asm volatile("" : "+v"(o[db][i]));  // one at a time: this may not cost the tile loop registers
        }
      if (__builtin_amdgcn_ballot_w64(poison && !all_nan) == 0) key1 = key0;
    }
}

// ---------------------------------------------------------------------------------------------
// Items of 128 query rows: 4 wavefronts, K and V tiles double buffered, loaded by all.
// ---------------------------------------------------------------------------------------------
template <class T>
constexpr int kDocsOff = T::ITEM_OFF + 16;
template <class T>
constexpr int kBadOff = kDocsOff<T> + 2 * T::BN * 4;
template <class T>
constexpr int kRowDocsOff = kBadOff<T> + 3 * 8;
template <class T>
constexpr int kMaskedLds = kRowDocsOff<T> + T::BM * 4;

// 64 ids -> LDS by one direct load of a dword a lane.
__device__ __forceinline__ void lds_dma_4(const int32_t* base, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds_addr), "v"(voff), "s"(base) : "memory");
}

// The rows of a wavefront, O^T / l, leave through LDS as whole rows (see store_out in attn_device.h): bf16 to out, or fp32 halves
// of rows to the workspace, from part_row on if that is not negative.  inv: 1 / l of the lane's row.
template <class T>
__device__ __forceinline__ void store_rows(const MaskedParams& p, const Lane<T>& L, const ItemU& it, int64_t part_row,
                                           const f32x16 (&o)[T::NDB], float inv, uint32_t stage) {
  typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
  if (part_row >= 0) {
    constexpr int CH = T::D / 8, RPS = 64 / CH;  // 16-byte chunks of half a row; half rows per store
    const int ch = L.lane & (CH - 1), r0 = L.lane / CH, row0 = L.wave * 32 + r0, n_valid = it.q_rows - row0;
    float* const dst = p.part_out + ((part_row + row0) * p.n_heads + it.head) * T::D + ch * 4;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int b = 0; b < T::NDB / 2; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int db = half * (T::NDB / 2) + b;
          const f32x4 f = {o[db][4 * g + 0] * inv, o[db][4 * g + 1] * inv, o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv};
          *(lds_u32x4*)(uintptr_t)(stage + (uint32_t)(L.l32 * (CH * 16) + (((8 * b + 2 * g + L.hh) ^ (L.l32 & (CH - 1))) * 16))) =
              __builtin_bit_cast(u32x4, f);
        }
      asm volatile("" ::: "memory");  // LDS serves a wavefront's instructions in order
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 32 / RPS; ++i) {
        const int r = r0 + i * RPS;
        const u32x4 w = *(lds_u32x4*)(uintptr_t)(stage + (uint32_t)(r * (CH * 16) + ((ch ^ (r & (CH - 1))) * 16)));
        if (i * RPS < n_valid)
          store_through(reinterpret_cast<u32x4*>(dst + (int64_t)(i * RPS) * p.n_heads * T::D + half * (T::D / 2)), w);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
    return;
  }
  constexpr int CH = T::ROW_B / 16, RPS = 64 / CH;
  const uint32_t wr = stage + (uint32_t)(L.l32 * T::ROW_B + L.hh * 8), wsw = (uint32_t)(L.l32 & (CH - 1)) * 16u;
#pragma unroll
  for (int db = 0; db < T::NDB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u32x2 w = {pack_bf16x2(o[db][4 * g + 0] * inv, o[db][4 * g + 1] * inv), pack_bf16x2(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv)};
      *(lds_u32x2*)(uintptr_t)(wr + ((uint32_t)((4 * db + g) * 16) ^ wsw)) = w;
    }
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  const int ch = L.lane & (CH - 1), r0 = L.lane / CH, row0 = L.wave * 32 + r0, n_valid = it.q_rows - row0;
  const int64_t row_b = (int64_t)p.n_heads * T::ROW_B;
  char* const dst = static_cast<char*>(p.out) + (int64_t)(it.q_start + row0) * row_b + (int64_t)it.head * T::ROW_B + ch * 16;
#pragma unroll
  for (int i = 0; i < 32 / RPS; ++i) {
    const int r = r0 + i * RPS;
    const u32x4 w = *(lds_u32x4*)(uintptr_t)(stage + (uint32_t)(r * T::ROW_B + ((ch ^ (r & (CH - 1))) * 16)));
    if (i * RPS < n_valid) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(dst + (int64_t)(i * RPS) * row_b));
  }
}

// slope * KEY + start, the constant within the instruction: as an operand the compiler keeps all 32 of a lane in registers.
template <int KEY>
__device__ __forceinline__ float linear_at(float slope, float start) {
  float x;
  asm("v_fmamk_f32 %0, %1, %3, %2" : "=v"(x) : "v"(slope), "v"(start), "n"(__builtin_bit_cast(int, (float)KEY)));
  return x;
}
template <int NKB>
__device__ __forceinline__ void linear_scores(f32x16 (&s)[NKB], float slope, float start) {
  static_for<0, NKB * 16>([&](auto kc) {
    constexpr int k = decltype(kc)::value;
    s[k / 16][k % 16] = linear_at<key_of(k / 16, k % 16)>(slope, start);
  });
}

// What a step does beside the softmax of an unmasked tile.
enum class Shape : int {
  kNone,
  kCap,     // sc are raw scores; their exponent is sc * (poly[0] + poly[1] sc^2 + poly[2] sc^4) - mc, see shape_scores
  kLinear,  // a bias that is linear over the tile: the accumulators of S^T(t+1) hold slope * key + start already, and those of
            // S^T(t), once their exponentials are taken, get what S^T(t+2) begins with (relative to the run's largest bias)
};

// One step: the exponentials of tile t beside the MFMAs of S^T(t+1) = K(t+1) Q^T and of O^T += V(t)^T P(t)^T, in the slots of
// tile_step (attn_device.h), then the maximum of S^T(t+1), with ABS that of its absolute values.
//   LSE: lx takes the sum of the fp32 probabilities.      issue: called behind every MFMA, for the loads of later tiles.
template <class T, int KOFF, int VOFF, int PD, Shape SHAPE, bool ABS, bool LSE, class Issue>
__device__ __forceinline__ void masked_step(const int (&va_)[T::NDB], const int (&ka_)[T::NKS], uint32_t (&pb)[T::NKB][8], const bf16x8 (&qf)[T::NKS],
                                            f32x16 (&o)[T::NDB], f32x16 (&sc)[T::NKB], f32x16 (&sn)[T::NKB], float c, float mc,
                                            const float (&poly)[3], float slope, float start, float& mx, float& lx, Issue&& issue) {
  using S = StepSlots<T>;
  constexpr int NQ = T::NQK, N = S::N;
  static_assert(T::NKB == 2, "two key blocks per tile");
  bf16x8 frag[PD];
  auto load_step = [&](auto jc) {
    constexpr int J = decltype(jc)::value;
    if constexpr (J >= NQ) {
      constexpr int j = J - NQ, kb = j / (2 * T::NDB), u = (j / T::NDB) % 2, db = j % T::NDB;
      lds_char* p0 = (lds_char*)(uintptr_t)(uint32_t)(va_[db] + VOFF + (32 * kb + 16 * u) * T::ROW_B);
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p0));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p0 + 8 * T::ROW_B));
      frag[J % PD] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      constexpr int ks = J / T::NKB, kb = J % T::NKB;
      frag[J % PD] = *(lds_bf16x8*)(uintptr_t)(uint32_t)(ka_[ks] + KOFF + kb * 32 * T::ROW_B);
    }
  };
  auto mfma = [&](auto jc) {
    constexpr int J = decltype(jc)::value;
    if constexpr (J >= NQ) {
      constexpr int j = J - NQ, kb = j / (2 * T::NDB), u = (j / T::NDB) % 2, db = j % T::NDB;
      const u32x4 pw = {pb[kb][4 * u], pb[kb][4 * u + 1], pb[kb][4 * u + 2], pb[kb][4 * u + 3]};
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[J % PD], __builtin_bit_cast(bf16x8, pw), o[db], 0, 0, 0);
    } else {
      constexpr int ks = J / T::NKB, kb = J % T::NKB;
      if constexpr (ks == 0 && SHAPE != Shape::kLinear) {
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        sn[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[J % PD], qf[ks], zero, 0, 0, 0);
      } else {
        sn[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[J % PD], qf[ks], sn[kb], 0, 0, 0);
      }
    }
  };
  auto exponent = [&](float x) {
    if constexpr (SHAPE == Shape::kCap) {
      const float z = x * x;
      return __builtin_fmaf(x, __builtin_fmaf(z, __builtin_fmaf(z, poly[2], poly[1]), poly[0]), -mc);
    } else {
      return __builtin_fmaf(x, c, -mc);
    }
  };
  float e0 = 0.f, e1 = 0.f;  // a pair is packed behind the exponentials of the next one
  auto unit = [&](auto kc) {
    constexpr int k = decltype(kc)::value;
    float f0 = 0.f, f1 = 0.f;
    if constexpr (k < S::UNITS) {
      constexpr int kb = k / 8, i = 2 * (k % 8);
      f0 = __builtin_amdgcn_exp2f(exponent(sc[kb][i]));
      f1 = __builtin_amdgcn_exp2f(exponent(sc[kb][i + 1]));
      if constexpr (SHAPE == Shape::kLinear) {
        sc[kb][i] = linear_at<key_of(kb, i)>(slope, start);
        sc[kb][i + 1] = linear_at<key_of(kb, i + 1)>(slope, start);
      }
    }
    if constexpr (k > 0) {
      SCHED_FENCE();
      pb[(k - 1) / 8][(k - 1) % 8] = pack_bf16x2(e0, e1);
      if constexpr (LSE) lx += e0 + e1;
    }
    e0 = f0;
    e1 = f1;
  };
  SCHED_FENCE();
  static_for<0, PD>([&](auto jc) { load_step(jc); });
  SCHED_FENCE();
  static_for<0, N>([&](auto jc) {
    constexpr int J = decltype(jc)::value;
    mfma(jc);
    if constexpr (J + PD < N) load_step(IC<J + PD>{});
    SCHED_FENCE();
    static_for<S::first_unit(J), S::first_unit(J + 1)>(unit);
    if constexpr (S::slot(S::UNITS - 1) == J) unit(IC<S::UNITS>{});
    issue(jc);
    if constexpr (J >= S::max_slot0) {
      constexpr int m = J - S::max_slot0, kb = m / 2, i = 8 * (m % 2);
#define DIT_MAX(O, C)                                                                                                               \
  if constexpr (m == 0)                                                                                                              \
    asm("v_max3_f32 %0, " O "%1" C ", " O "%2" C ", " O "%3" C "\n\tv_max3_f32 %0, %0, " O "%4" C ", " O "%5" C                    \
        "\n\tv_max3_f32 %0, %0, " O "%6" C ", " O "%7" C "\n\tv_max3_f32 %0, %0, %0, " O "%8" C                                  \
        : "=&v"(mx)                                                                                                                  \
        : "v"(sn[0][0]), "v"(sn[0][1]), "v"(sn[0][2]), "v"(sn[0][3]), "v"(sn[0][4]), "v"(sn[0][5]), "v"(sn[0][6]), "v"(sn[0][7]));  \
  else                                                                                                                               \
    asm("v_max3_f32 %0, %0, " O "%1" C ", " O "%2" C "\n\tv_max3_f32 %0, %0, " O "%3" C ", " O "%4" C                              \
        "\n\tv_max3_f32 %0, %0, " O "%5" C ", " O "%6" C "\n\tv_max3_f32 %0, %0, " O "%7" C ", " O "%8" C                        \
        : "+v"(mx)                                                                                                                   \
        : "v"(sn[kb][i]), "v"(sn[kb][i + 1]), "v"(sn[kb][i + 2]), "v"(sn[kb][i + 3]), "v"(sn[kb][i + 4]), "v"(sn[kb][i + 5]),        \
          "v"(sn[kb][i + 6]), "v"(sn[kb][i + 7]))
      if constexpr (ABS) {
        DIT_MAX("|", "|");
      } else {
        DIT_MAX("", "");
      }
#undef DIT_MAX
    }
    SCHED_FENCE();
  });
  mx = max_with_other_half(mx);
  SCHED_FENCE();
}

// Workgroups on a compute unit: what the registers allow.
template <int D, bool CAP, bool LSE>
constexpr int kMaskedWaves = D == 64 && !(CAP && LSE) ? 3 : 2;

// The kernel works a tile ahead, as the unmasked 128-row kernel: the scores of the next tile are contracted beside the softmax of
// this one.  Most tiles are touched by no mask; runs of them have a loop of their own, in which a cap and a bias cost their few
// instructions a score beside the MFMAs.  What else shapes and masks a tile's scores stands between two steps.
// us on MI355X, with the three parts of a tile in turn / now:  20506 rows x 24 heads, D 128, unmasked 5387 / 4330 (1190 TFLOP/s, the
// unmasked 128-row kernel 4220), cap 6888 / 5060, bias 6237 / 4580, causal 2603 / 2130;  4352 x 24 x 6, D 64, unmasked 790 / 690,
// bias 987 / 766, padded documents of three 559 / 393.  Bound by power (1.7 GHz) with both pipes of a SIMD over half busy; the
// padded documents by vector instructions, half of their tiles being at an edge of a document or around the rows' own places.
// That cap is of scores under a quarter of it, which take the polynomial alone.  One score past that in 32 rows and 64 keys and the
// wavefront computes both forms of all of them between two steps, an exponential and a reciprocal each:  unmasked / small / large
// 4380 / 5150 / 8300 at D 128, 696 / 870 / 1683 at D 64.  Cap and bias together are shaped between two steps too:  5860 with small
// scores and 8170 with large ones, 1022 and 1598.
// 128 rows and not 64 or 256: two workgroups of four wavefronts fill a compute unit's registers and 130 of its 160 KB LDS.
template <class T, bool CAP, bool BIAS, bool LSE>
__global__ void __attribute__((amdgpu_flat_work_group_size(T::NT, T::NT), amdgpu_waves_per_eu(kMaskedWaves<T::D, CAP, LSE>, kMaskedWaves<T::D, CAP, LSE>)))
masked_attn_kernel(MaskedParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
  lds_char* smem = (lds_char*)smem_generic;
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  const int tid = threadIdx.x;
  // Per-lane constants are recomputed where they are needed; kept live through the tile loop they are spilled.
  auto fresh_lane = [&]() {
    int x = tid;
    asm volatile("" : "+v"(x));
    Lane<T> l;
    l.init(x, p.k_stride_b);
    return l;
  };
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // The item: heads fastest, so that with a multiple of eight heads an XCD keeps to its own ones; the last query tiles first,
  // which see the most keys under a causal mask.
  const MaskedSeq& sq = find_seq<&MaskedSeq::first>(p, p.n, blockIdx.x);
  const int n_heads = p.n_heads, lq = sq.q_len, lk = sq.kv_len;
  uint32_t local = blockIdx.x - sq.first;
  ItemU it;
  it.part = (int)(local % (uint32_t)sq.parts);
  local /= (uint32_t)sq.parts;
  it.head = (int)(local % (uint32_t)n_heads);
  const int m0 = ((lq + T::BM - 1) / T::BM - 1 - (int)(local / (uint32_t)n_heads)) * T::BM;
  static_assert(T::BM == kMaskedBlockM, "items as the host counts them");
  it.q_start = sq.q_start + m0;
  it.q_rows = lq - m0 < T::BM ? lq - m0 : T::BM;
  it.kv_start = sq.kv_start;

  // Keys under lim are all that any row sees; a row sees keys under its klim.
  const int pos0 = m0 + lk - lq;
  int lim = lk;
  if (p.causal) {
    const int last = pos0 + it.q_rows > sq.prefix ? pos0 + it.q_rows : sq.prefix;
    lim = last < lk ? last : lk;
  }
  auto row_limit = [&](int row) {
    if (!p.causal) return lim;
    const int k = pos0 + row + 1 > sq.prefix ? pos0 + row + 1 : sq.prefix;
    return k < lim ? k : lim;
  };
  // This lane's query row, or the last one.
  auto query_row = [&]() {
    int x = tid;
    asm volatile("" : "+v"(x));
    const int row = (x >> 6) * 32 + (x & 31);
    return row < it.q_rows ? row : it.q_rows - 1;
  };
  const int klim_first = row_limit(0);

  LiveTiles tiles;
  tiles.ranges = nullptr;
  tiles.base = -64;
  tiles.live = tiles.pure = 0;
  const int nt = lim > 0 ? (lim + T::BN - 1) / T::BN : 0;
  const int64_t part_end = ((int64_t)it.part + 1) * p.part_tiles;
  int t0 = nt;
  if ((int64_t)it.part * p.part_tiles < nt) t0 = it.part * p.part_tiles;
  tiles.end = part_end < nt ? (int)part_end : nt;
  const bool have_docs = p.q_doc != nullptr;
  const int32_t* kdoc = nullptr;
  if (have_docs) {
    kdoc = p.k_doc + sq.kv_start;
    const int row = query_row();  // a row's id is read back by the wavefront that wrote it
    *(lds_u32*)(uintptr_t)(lds + kRowDocsOff<T> + row * 4) = (uint32_t)p.q_doc[it.q_start + row];
    const DocTile a = doc_range(p.q_doc + it.q_start, it.q_rows < 64 ? it.q_rows : 64);
    const DocTile b = it.q_rows > 64 ? doc_range(p.q_doc + it.q_start + 64, it.q_rows - 64) : a;
    tiles.mine.lo = a.lo < b.lo ? a.lo : b.lo;
    tiles.mine.hi = a.hi > b.hi ? a.hi : b.hi;
    tiles.mine.any_lo = a.any_lo < b.any_lo ? a.any_lo : b.any_lo;
    tiles.ranges = p.doc_tiles + sq.tile0;
  }
  t0 = tiles.next(t0);

  // The id of this lane's row, and the keys that the row sees are under the limit.
  auto row_mask = [&](int row, int& doc) {
    doc = have_docs ? (int)*(lds_u32*)(uintptr_t)(lds + kRowDocsOff<T> + row * 4) : 0;
    return doc < 0 ? 0 : row_limit(row);
  };

  f32x16 o[T::NDB];
#pragma unroll
  for (int db = 0; db < T::NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  RowState r = {kNoReference, 0.f, 0.f};

  if (t0 < tiles.end) {
    const int kv_head = it.head / p.group;
    const char* kbase = static_cast<const char*>(p.k) + (int64_t)it.kv_start * p.k_stride_b + (int64_t)kv_head * T::ROW_B;
    const char* vbase = static_cast<const char*>(p.v) + (int64_t)it.kv_start * p.v_stride_b + (int64_t)kv_head * T::ROW_B;
    const float c = CAP ? 1.f : p.c_log2;
    const float slope = BIAS ? p.slopes[it.head] * 1.44269504088896340736f / c : 0.f;
    const uint32_t lds_wave = lds + (uint32_t)wave * 1024u;
    const TailRows tail = tail_rows<T>(lim);
    uint32_t kvoff, vvoff;
    {
      const Lane<T> L = fresh_lane();
      kvoff = L.kvoff;
      vvoff = (uint32_t)L.lrow * (uint32_t)p.v_stride_b + (uint32_t)L.vcol;
    }
    // Some pair of a row of the item and a key of tile t is dead.  Asked before the walk over the tiles goes on.
    auto needs_mask = [&](int t) {
      return (t == nt - 1 && tail.hi - tail.lo != T::BN) || klim_first < tile_first_key<T>(t, lim) + T::BN || !tiles.is_pure(t);
    };
    // Whole tiles (keys under a tile are loaded as a tile of the last 64 ones, or, where all of them are under one, in the prologue).
    auto load_k = [&](int t, int slot) {
      const int key0 = tile_first_key<T>(t, lim);
      const char* base = kbase + (int64_t)key0 * p.k_stride_b;
#pragma unroll
      for (int i = 0; i < T::LPT; ++i)
        lds_dma_16(base + (int64_t)(i * T::GROUP) * p.k_stride_b, kvoff, lds_wave + T::K_OFF + slot * T::TILE_B + i * T::NWAVES * 1024);
      if (have_docs && wave == 0) lds_dma_4(kdoc + key0, (uint32_t)(tid * 4), lds + kDocsOff<T> + slot * (T::BN * 4));
    };
    auto load_v = [&](int t, int slot) {
      const char* base = vbase + (int64_t)tile_first_key<T>(t, lim) * p.v_stride_b;
#pragma unroll
      for (int i = 0; i < T::LPT; ++i)
        lds_dma_16(base + (int64_t)(i * T::GROUP) * p.v_stride_b, vvoff, lds_wave + T::V_OFF + slot * T::TILE_B + i * T::NWAVES * 1024);
    };

    // Q goes through slots that the first tiles do not need yet.
    const uint32_t spare = lds + (wave < 2 ? T::K_OFF : T::V_OFF) + T::TILE_B + (uint32_t)(wave % 2) * (32 * T::ROW_B);
    static_assert(T::TILE_B == 2 * 32 * T::ROW_B, "two wavefronts' rows in a tile");
    bool masked0 = needs_mask(t0);
    {
      const Lane<T> L = fresh_lane();
      q_rows_load<T>(p, L, it, p.q_stride_b, (int64_t)it.head * T::ROW_B, spare);
      if (lim >= T::BN) {
        load_k(t0, 0);
        load_v(t0, 0);
      } else {
        tile_load_one<T>(kbase, p.k_stride_b, 0, lim, L.lrow, L.kcol, kvoff, smem, T::K_OFF, wave);
        if (have_docs && wave == 0) lds_dma_4(kdoc, (uint32_t)(tid < lim ? tid : lim - 1) * 4u, lds + kDocsOff<T>);
        tile_load_one<T>(vbase, p.v_stride_b, 0, lim, L.lrow, L.vcol, vvoff, smem, T::V_OFF, wave);
      }
    }
    if (tid < 6) *(lds_u32*)(uintptr_t)(lds + kBadOff<T> + tid * 4) = 0;
    int t1 = tiles.next(t0 + 1);
    bool masked1 = t1 < tiles.end && needs_mask(t1);
    int t2 = tiles.next(t1 + 1);
    bool masked2 = t2 < tiles.end && needs_mask(t2);
    wait_loads_but<T::LPT>();  // V is awaited before its step
    bf16x8 qf[T::NKS];
    q_rows_read<T>(p, fresh_lane(), spare, qf);
    wg_barrier();
    int ka[T::NKS], va[T::NDB];
    fresh_lane().operand_addrs(lds, lds, ka, va);
    int turn = 0;  // of the bad-key masks
    bool poison = false;
    float mx = 0.f;
    f32x16 sa[T::NKB], sb[T::NKB];
    uint32_t pb[T::NKB][8];

    // Scores of tile t, from S^T to shaped ones with the dead ones -inf, and their maximum mx.  Before, mx is the maximum of the
    // raw scores, with a cap that of their absolute values: if it is small, its capped value serves as the maximum, which it
    // exceeds by at most 2^60 in the probabilities (p.small); else the shaped scores are gone through.
    auto is_small = [&]() { return __builtin_amdgcn_ballot_w64(!(mx <= p.small)) == 0; };
    // pos - first key of tile t - 4 hh
    auto distance = [&](int t) { return pos0 + query_row() - tile_first_key<T>(t, lim) - 4 * half_of(tid); };
    auto finish = [&](f32x16(&s)[T::NKB], int t, int slot, bool masked) {
      const int key0 = tile_first_key<T>(t, lim);
      const bool small = CAP && is_small();
      if constexpr (CAP || BIAS) shape_scores<T::NKB, CAP, BIAS>(s, p, small, slope, BIAS ? distance(t) : 0);
      if (masked) {
        int doc;
        const int hh = half_of(tid), klim = row_mask(query_row(), doc);
        const int lo = t == nt - 1 ? tail.lo : 0, n = klim - key0 - lo;
        const LaneMask m = {lo - 4 * hh, n > 0 ? (unsigned)n : 0u};
        mask_scores<T::NKB>(s, m, have_docs, lds + kDocsOff<T> + slot * (T::BN * 4), doc, hh);
      }
      if (BIAS || masked || (CAP && !small)) {
        scores_ready<T>(s);
        mx = tile_max<T>(s);
      } else if constexpr (CAP) {
        mx = small_cap(p, mx);
      }
    };
    // Behind the loads of V of a masked tile, before the barrier: this wavefront's rows of it become finite.
    auto clean_v = [&](int slot) {
      const uint32_t found = make_finite<T::LPT>(lds_wave + T::V_OFF + slot * T::TILE_B + (tid & 63) * 16, T::NWAVES * 1024);
      if (found != 0) {
        const int lrow = fresh_lane().lrow;
#pragma unroll
        for (int i = 0; i < T::LPT; ++i) {
          const int row = i * T::GROUP + lrow;
          if (found >> i & 1)
            __hip_atomic_fetch_or((lds_u32*)(uintptr_t)(lds + kBadOff<T> + (uint32_t)turn * 8u + (uint32_t)(row >> 5) * 4u), 1u << (row & 31),
                                  __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
      }
    };
    // Behind that barrier: whether a row of this lane sees one of those keys.  Clears the mask of the tile after the next.
    auto look_bad = [&](const f32x16(&s)[T::NKB], bool masked) {
      if (masked) {
        const uint32_t at = lds + kBadOff<T> + (uint32_t)turn * 8u;
        const uint64_t bad = mask_of_words(__builtin_amdgcn_readfirstlane(*(lds_u32*)(uintptr_t)at),
                                           __builtin_amdgcn_readfirstlane(*(lds_u32*)(uintptr_t)(at + 4)));
        if (bad != 0) poison |= sees<T::NKB>(s, bad, half_of(tid));
      }
      const int clear = turn == 0 ? 2 : turn - 1;
      if (tid < 2) *(lds_u32*)(uintptr_t)(lds + kBadOff<T> + (uint32_t)clear * 8u + tid * 4) = 0;
      turn = turn == 2 ? 0 : turn + 1;
    };
    auto raise = [&]() {
      const bool grow = (mx - r.m_ref) * c > kRescaleLog2;
      if (__builtin_amdgcn_ballot_w64(grow) != 0) {
        const float m_new = grow ? mx : r.m_ref;
        const float alpha = __builtin_amdgcn_exp2f((r.m_ref - m_new) * c);
        r.m_ref = m_new;
        r.l *= alpha;
        if constexpr (LSE) r.lx *= alpha;
#pragma unroll
        for (int db = 0; db < T::NDB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      }
    };

    if (t1 < tiles.end) load_k(t1, 1);
    mfma_stream<T, false, 0, T::NQK, kPrefetch>(smem, va, ka, pb, qf, o, sa);
    if constexpr (CAP) {
      mx = __builtin_inff();  // not known of the first tile
    } else {
      scores_ready<T>(sa);
      mx = tile_max<T>(sa);
    }

    // Tiles under free_end need no mask but for ids.  In a run of such tiles, whose ids agree too, a step has no tests and loads
    // from running pointers, spread behind its MFMAs.
    const int free_end = klim_first / T::BN < tiles.end ? klim_first / T::BN : tiles.end;
    constexpr int NLOAD = 2 * T::LPT, EVERY = (T::NQK + T::NPV) / 2 / NLOAD;
    static_assert(EVERY >= 1, "a step's loads fit its slots");
    const char *kp = kbase, *vp = vbase;
    const int64_t k_step = (int64_t)T::BN * p.k_stride_b, v_step = (int64_t)T::BN * p.v_stride_b;
    constexpr Shape SHAPE = BIAS ? (CAP ? Shape::kNone : Shape::kLinear) : CAP ? Shape::kCap : Shape::kNone;
    // With kLinear all keys of a run lie on one side of all rows, and its bias is side * (key - pos).  An accumulator that began
    // with that would round every product at the size of the bias, so within a run scores and their reference are relative to
    // the row's largest bias there, of key `anchor`: those that count then are small.
    float side = 0.f;
    int anchor = 0;
    auto anchor_bias = [&]() { return side * (float)(anchor - pos0 - query_row()); };
    auto linear_start = [&](int t) { return side * (float)(t * T::BN + 4 * half_of(tid) - anchor); };
    // A step from t (scores raw with kCap, else shaped, in sc; K(t + 1) and V(t) on their way) to t + 1 (in sn, shaped with
    // kLinear, else raw).
    auto run_step = [&](auto uc, f32x16(&sc)[T::NKB], f32x16(&sn)[T::NKB]) {
      constexpr int U = decltype(uc)::value;
      wait_loads();
      wg_barrier();
      float poly[3] = {1.f, 0.f, 0.f};
      if constexpr (SHAPE == Shape::kCap) {
        if (is_small()) {
#pragma unroll
          for (int i = 0; i < 3; ++i) poly[i] = p.poly[i];
          mx = small_cap(p, mx);
        } else {
          shape_scores<T::NKB, CAP, false>(sc, p, false, 0.f, 0);
          scores_ready<T>(sc);
          mx = tile_max<T>(sc);
        }
      }
      const float start = SHAPE == Shape::kLinear ? linear_start(t0 + 2) : 0.f;
      raise();
      const float mc = __builtin_fmaxf(r.m_ref * c, -3.0e38f);
      masked_step<T, (1 - U) * T::TILE_B, U * T::TILE_B, T::D == 64 && SHAPE == Shape::kLinear ? 3 : kPrefetch, SHAPE, CAP, LSE>(
          va, ka, pb, qf, o, sc, sn, c, mc, poly, side, start, mx, r.lx, [&](auto jc) {
            constexpr int J = decltype(jc)::value;
            if constexpr (J % EVERY == EVERY / 2 && J / EVERY < NLOAD) {
              constexpr int j = J / EVERY, i = j % T::LPT;
              if constexpr (j < T::LPT)
                lds_dma_16_at<T::K_OFF + U * T::TILE_B + i * T::NWAVES * 1024>(kp + (int64_t)(i * T::GROUP) * p.k_stride_b, kvoff, lds_wave);
              else
                lds_dma_16_at<T::V_OFF + (1 - U) * T::TILE_B + i * T::NWAVES * 1024>(vp + (int64_t)(i * T::GROUP) * p.v_stride_b, vvoff, lds_wave);
            }
          });
      kp += k_step;
      vp += v_step;
      r.l += row_sum<T>(pb);
      asm volatile("" : "+v"(r.l));
      ++t0;
    };
    int slot = 0;  // of K(t0) and V(t0); ka and va point there
    auto turn_slots = [&]() {
#pragma unroll
      for (int db = 0; db < T::NDB; ++db) va[db] ^= T::TILE_B;
      slot ^= 1;
    };
    auto turn_k = [&]() {
#pragma unroll
      for (int ks = 0; ks < T::NKS; ++ks) ka[ks] ^= T::TILE_B;
    };
    while (t1 < tiles.end) {
      // Here the scores of t0 are raw, in sa; K(t1) and V(t0) are on their way.
      bool shaped = false;
      if (slot == 0 && !masked0) {
        int run_end = free_end;
        if (tiles.ranges != nullptr) {
          const int rest = t0 >= tiles.base ? t0 + (int)__builtin_ctzll(~((tiles.live & tiles.pure) >> (t0 - tiles.base)) | 1ull << 63) : t0;
          run_end = rest < run_end ? rest : run_end;
        }
        if constexpr (SHAPE == Shape::kLinear) {
          const int left_end = pos0 >= 0 ? (pos0 + 1) / T::BN : 0;  // tiles whose keys are all up to the first row's place
          const bool right = t0 * T::BN >= pos0 + it.q_rows - 1;    // all from the last one's on
          side = right ? -slope : slope;
          if (!right && left_end < run_end) run_end = left_end;
        }
        if (t0 + 3 < run_end) {
          kp = kbase + (int64_t)(t0 + 2) * k_step;
          vp = vbase + (int64_t)(t0 + 1) * v_step;
          if constexpr (SHAPE == Shape::kLinear) {
            anchor = side > 0.f ? run_end * T::BN - 1 : t0 * T::BN;
            r.m_ref -= anchor_bias();
            linear_scores<T::NKB>(sb, side, linear_start(t0));
#pragma unroll
            for (int kb = 0; kb < T::NKB; ++kb) sa[kb] += sb[kb];
            scores_ready<T>(sa);
            mx = tile_max<T>(sa);
            linear_scores<T::NKB>(sb, side, linear_start(t0 + 1));
          }
          do {
            if constexpr (SHAPE == Shape::kNone && BIAS) finish(sa, t0, 0, false);
            run_step(IC<0>{}, sa, sb);
            if constexpr (SHAPE == Shape::kNone && BIAS) finish(sb, t0, 0, false);
            run_step(IC<1>{}, sb, sa);
          } while (t0 + 3 < run_end);
          if constexpr (SHAPE == Shape::kLinear) {
            const float base = anchor_bias();
            r.m_ref += base;
            mx += base;
#pragma unroll
            for (int kb = 0; kb < T::NKB; ++kb)
#pragma unroll
              for (int i = 0; i < 16; ++i) sa[kb][i] += base;
            shaped = true;
          }
          t1 = t0 + 1;
          t2 = tiles.next(t1 + 1);
          masked0 = masked1 = false;
          masked2 = t2 < tiles.end && needs_mask(t2);
        }
      }
      if (!shaped) finish(sa, t0, slot, masked0);
      const int t3 = tiles.next(t2 + 1);
      const bool masked3 = t3 < tiles.end && needs_mask(t3);
      wait_loads();
      if (masked0) clean_v(slot);
      wg_barrier();
      if (t2 < tiles.end) load_k(t2, slot);
      load_v(t1, slot ^ 1);
      look_bad(sa, masked0);
      raise();
      const float mc = __builtin_fmaxf(r.m_ref * c, -3.0e38f);
      turn_k();
      masked_step<T, 0, 0, kPrefetch, Shape::kNone, CAP, LSE>(va, ka, pb, qf, o, sa, sb, c, mc, p.poly, 0.f, 0.f, mx, r.lx, [](auto) {});
      turn_slots();
      r.l += row_sum<T>(pb);
      asm volatile("" : "+v"(r.l));
#pragma unroll
      for (int kb = 0; kb < T::NKB; ++kb) sa[kb] = sb[kb];
      t0 = t1;
      t1 = t2;
      t2 = t3;
      masked0 = masked1;
      masked1 = masked2;
      masked2 = masked3;
    }
    finish(sa, t0, slot, masked0);
    wait_loads();
    if (masked0) clean_v(slot);
    wg_barrier();
    look_bad(sa, masked0);
    masked_softmax<T::NKB, T::NDB, LSE>(sa, mx, c, pb, o, r);
    mfma_stream<T, true, 0, 0, kPrefetch>(smem, va, ka, pb, qf, o, sa);
    r.l += row_sum<T>(pb);
    poison = either_half(poison);
    if (__builtin_amdgcn_ballot_w64(poison) != 0) {
      const int k0 = it.part * p.part_tiles * T::BN;
      int doc;
      const int klim = row_mask(query_row(), doc);
      add_not_finite<T>(p, vbase, kdoc, k0, tiles.end * T::BN < lim ? tiles.end * T::BN : lim, T::BN, T::BN, klim, doc, half_of(tid), poison, o);
    }
    // The rows are staged in the K buffers, which nobody reads behind the last barrier.
  }

  const float l = r.l + __shfl_xor(r.l, 32), lx = r.lx + __shfl_xor(r.lx, 32);
  const bool any = l > 0.f || l != l;
  const int64_t part_row = sq.parts > 1 ? sq.part_row + (int64_t)it.part * lq + m0 : -1;
  store_rows<T>(p, fresh_lane(), it, part_row, o, any ? 1.f / l : 0.f, lds + T::K_OFF + (uint32_t)wave * (32 * T::ROW_B));
  if constexpr (LSE) {
    const int qrow = wave * 32 + (tid & 31);
    if (qrow < it.q_rows && (tid & 32) == 0) {
      const float c = CAP ? 1.f : p.c_log2;
      float* dst = part_row >= 0 ? p.part_lse + (part_row + qrow) * n_heads : p.lse + (int64_t)(it.q_start + qrow) * n_heads;
      if (part_row >= 0 || p.lse != nullptr) dst[it.head] = any ? kLn2 * (r.m_ref * c + __builtin_amdgcn_logf(lx)) : -__builtin_inff();
    }
  }
#endif
}

// ---------------------------------------------------------------------------------------------
// Few query rows (one new token, say): every (row, query head of a key head's group) is a column, at most 32 of them, so that
// K and V are read once for the whole group.  Bound by reading them.  Eight wavefronts take blocks of keys in turn, each with
// loads, LDS and softmax state of its own and no barrier until the end, when their results are joined.  A wavefront's K buffer
// takes the next block as soon as the scores are contracted, its V buffer as soon as O^T is: two wavefronts on a SIMD keep both
// in flight, 128 KB a compute unit.
// us on MI355X, four wavefronts with two stages of K and V each / this, unsplit:  one row of 8 heads, D 128, against 448 keys 10.6 /
// 7.5, 2048 30.9 / 15.6, 20506 266 / 131;  eight rows against 41800 keys in all, 8 key heads for 24, split: 41.6 / 28.7 (5.7 TB/s).
// ---------------------------------------------------------------------------------------------
template <int D>
struct FewRows {
  static constexpr int KEYS = 4096 / D;                    // of a block: 8 KB of K and of V
  using T = Tile<D, 4, KEYS>;
  static constexpr int WAVES = 8;
  static constexpr int BLOCK_B = KEYS * T::ROW_B;
  static constexpr int WAVE_B = 2 * BLOCK_B;               // [K, V]
  static constexpr int DOCS_OFF = WAVES * WAVE_B;          // [wave][2][KEYS] ids
  static constexpr int DOCS_B = KEYS * 4;
  static constexpr int STATE_OFF = DOCS_OFF + WAVES * 2 * DOCS_B;  // [m, l, lx][wave][column]
  static constexpr int LDS_BYTES = STATE_OFF + 3 * WAVES * 32 * 4;
  static constexpr int N = KEYS / T::RPI;                  // load instructions of a block of K or V
  static_assert(32 * D * 4 <= WAVE_B, "a wavefront's result fits its buffers");
};

template <int D, bool CAP, bool BIAS>
__global__ void __attribute__((amdgpu_flat_work_group_size(512, 512), amdgpu_waves_per_eu(2, 2))) masked_few_rows_kernel(MaskedParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
  using F = FewRows<D>;
  using T = typename F::T;
  extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
  lds_char* smem = (lds_char*)smem_generic;
  const uint32_t lds = (uint32_t)(uintptr_t)smem;
  const int tid = threadIdx.x;
  Lane<T> L;
  L.init(tid, p.k_stride_b);
  const int wave = L.wave, hh = L.hh;

  const MaskedSeq& sq = find_seq<&MaskedSeq::first>(p, p.n, blockIdx.x);
  const int lq = sq.q_len, lk = sq.kv_len, group = p.group, n_heads = p.n_heads;
  uint32_t local = blockIdx.x - sq.first;
  const int part = (int)(local % (uint32_t)sq.parts), kv_head = (int)(local / (uint32_t)sq.parts);
  const int n_cols = lq * group;
  // This lane's column, or the last one, as its row and head.
  auto column = [&](int& head) {
    int x = tid;
    asm volatile("" : "+v"(x));
    const int c = (x & 31) < n_cols ? (x & 31) : n_cols - 1, row = c / group;
    head = kv_head * group + (c - row * group);
    return row;
  };

  const int pos0 = lk - lq;
  auto row_limit = [&](int i) {
    if (!p.causal) return lk;
    const int k = pos0 + i + 1 > sq.prefix ? pos0 + i + 1 : sq.prefix;
    return k < lk ? k : lk;
  };
  const int lim = row_limit(lq - 1), klim_first = row_limit(0);

  LiveTiles tiles;
  tiles.ranges = nullptr;
  tiles.base = -64;
  tiles.live = tiles.pure = 0;
  const int nt = lim > 0 ? (lim + 63) / 64 : 0;
  const int64_t part_end = ((int64_t)part + 1) * p.part_tiles;
  int t0 = nt;
  if ((int64_t)part * p.part_tiles < nt) t0 = part * p.part_tiles;
  tiles.end = part_end < nt ? (int)part_end : nt;
  const bool have_docs = p.q_doc != nullptr;
  const int32_t* kdoc = nullptr;
  if (have_docs) {
    kdoc = p.k_doc + sq.kv_start;
    tiles.mine = doc_range(p.q_doc + sq.q_start, lq);
    tiles.ranges = p.doc_tiles + sq.tile0;
  }
  // The id of this lane's row, and the keys that the row sees are under the limit.
  auto row_mask = [&](int& doc) {
    int head;
    const int row = column(head);
    doc = have_docs ? p.q_doc[sq.q_start + row] : 0;
    return doc < 0 ? 0 : row_limit(row);
  };
  // Blocks of keys; this wavefront's are wave, wave + 8, ... of those in live tiles.
  constexpr int BPT = 64 / F::KEYS;  // blocks of a tile
  const int all_blocks = (lim + F::KEYS - 1) / F::KEYS, n_blocks = tiles.end * BPT < all_blocks ? tiles.end * BPT : all_blocks;
  auto next_block = [&](int b) {
    while (b < n_blocks) {
      const int t = tiles.next(b / BPT);
      if (t == b / BPT) return b;
      b += (BPT * t - b + F::WAVES - 1) & ~(F::WAVES - 1);
    }
    return n_blocks;
  };
  const int first_block = t0 * BPT + ((wave - t0 * BPT) & (F::WAVES - 1));

  f32x16 o[T::NDB];
#pragma unroll
  for (int db = 0; db < T::NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;
  RowState r = {kNoReference, 0.f, 0.f};
  const float c = CAP ? 1.f : p.c_log2;
  const uint32_t kbuf = lds + (uint32_t)wave * F::WAVE_B, vbuf = kbuf + F::BLOCK_B, docs = lds + F::DOCS_OFF + (uint32_t)wave * (2 * F::DOCS_B);

  int block = t0 < tiles.end ? next_block(first_block) : n_blocks;
  if (block < n_blocks) {
    const char* kbase = static_cast<const char*>(p.k) + (int64_t)sq.kv_start * p.k_stride_b + (int64_t)kv_head * T::ROW_B;
    const char* vbase = static_cast<const char*>(p.v) + (int64_t)sq.kv_start * p.v_stride_b + (int64_t)kv_head * T::ROW_B;
    int head;
    const int row = column(head);
    const float slope = BIAS ? p.slopes[head] * 1.44269504088896340736f / c : 0.f;
    const int at0 = BIAS ? pos0 + row - 4 * hh : 0;
    // Lane offsets of the load instructions, RPI rows each: a V row's chunk order has a period of one, a K row's of KN.
    constexpr int KN = 16 / T::RPI;
    uint32_t koff[KN], voff;
    {
      const int at = L.lane % T::CPR, q = L.lane / T::CPR;  // chunk and row
#pragma unroll
      for (int i = 0; i < KN; ++i) koff[i] = (uint32_t)q * (uint32_t)p.k_stride_b + (uint32_t)((at ^ T::swz_k(i * T::RPI + q)) * 16);
      voff = (uint32_t)q * (uint32_t)p.v_stride_b + (uint32_t)((at ^ T::swz_v(q)) * 16);
      static_assert(T::swz_k(16) == T::swz_k(0) && T::swz_v(T::RPI) == T::swz_v(0), "periods");
    }
    auto load_rows = [&](auto is_k, const char* base, int64_t stride_b, int key0, uint32_t buf) {
      constexpr bool K = decltype(is_k)::value != 0;
      const char* b = base + (int64_t)key0 * stride_b;
      if (key0 + F::KEYS <= lim) {
#pragma unroll
        for (int i = 0; i < F::N; ++i) lds_dma_16(b + (int64_t)(i * T::RPI) * stride_b, K ? koff[i % KN] : voff, buf + i * 1024);
      } else {  // rows past the last key re-read it (they are dead)
        int lane = tid & 63;
        asm volatile("" : "+v"(lane));
        const int at = lane % T::CPR, q = lane / T::CPR, last = lim - 1 - key0;
#pragma unroll
        for (int i = 0; i < F::N; ++i) {
          const int rr = i * T::RPI + q, from = rr < last ? rr : last;
          lds_dma_16(b, (uint32_t)from * (uint32_t)stride_b + (uint32_t)((at ^ (K ? T::swz_k(rr) : T::swz_v(rr))) * 16), buf + i * 1024);
        }
      }
    };
    int turn = 0;  // of the ids
    auto load_k = [&](int b, int to) {
      const int key0 = b * F::KEYS;
      load_rows(IC<1>{}, kbase, p.k_stride_b, key0, kbuf);
      if (have_docs) {
        const int last = lim - 1 - key0, k = L.lane < last ? L.lane : last;
        if (L.lane < F::KEYS) lds_dma_4(kdoc + key0, (uint32_t)k * 4u, docs + (uint32_t)(to * F::DOCS_B));
      }
    };
    load_k(block, 0);
    load_rows(IC<0>{}, vbase, p.v_stride_b, block * F::KEYS, vbuf);

    bf16x8 qf[T::NKS];
    {
      const char* qp = static_cast<const char*>(p.q) + (int64_t)(sq.q_start + row) * p.q_stride_b + (int64_t)head * T::ROW_B + hh * 16;
#pragma unroll
      for (int ks = 0; ks < T::NKS; ++ks) {
        u32x4 w = *reinterpret_cast<const u32x4*>(qp + ks * 32);
        if (p.negate) w ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
        qf[ks] = __builtin_bit_cast(bf16x8, w);
      }
    }
    int ka[T::NKS], va[T::NDB];
    L.operand_addrs(kbuf - T::K_OFF, vbuf - T::V_OFF, ka, va);
    bool poison = false;
    while (block < n_blocks) {
      const int key0 = block * F::KEYS;
      const bool masked = klim_first < key0 + F::KEYS || !tiles.is_pure(block / BPT);
      const int next = next_block(block + F::WAVES);
      wait_loads_but<F::N>();  // V may be outstanding
      f32x16 s[T::NKB];
      uint32_t pb[T::NKB][8];
      mfma_stream<T, false, 0, T::NQK, kPrefetch>(smem, va, ka, pb, qf, o, s);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K has been read
      if (next < n_blocks) load_k(next, turn ^ 1);
      if constexpr (CAP || BIAS) shape_scores<T::NKB, CAP, BIAS>(s, p, false, slope, at0 - key0);
      if (masked) {
        int doc;
        const int n = row_mask(doc) - key0;
        const LaneMask m = {-4 * hh, n > 0 ? (unsigned)n : 0u};
        mask_scores<T::NKB>(s, m, have_docs, docs + (uint32_t)(turn * F::DOCS_B), doc, hh);
      }
#pragma unroll
      for (int kb = 0; kb < T::NKB; ++kb) asm volatile("s_nop 11" : "+v"(s[kb]));  // as scores_ready
      const float mx = tile_max<T>(s);
      masked_softmax<T::NKB, T::NDB, true>(s, mx, c, pb, o, r);
      // V has landed when only the next K (and its ids) may be outstanding.
      if (next >= n_blocks) wait_loads();
      else if (have_docs) wait_loads_but<F::N + 1>();
      else wait_loads_but<F::N>();
      if (masked) {
        uint64_t bad = 0;
        const uint32_t found = make_finite<F::N>(vbuf + (uint32_t)L.lane * 16u, 1024);
        if (__builtin_amdgcn_ballot_w64(found != 0) != 0) {
#pragma unroll
          for (int i = 0; i < F::N; ++i) {
            const uint64_t rows = __builtin_amdgcn_ballot_w64((found >> i & 1) != 0);
#pragma unroll
            for (int k = 0; k < T::RPI; ++k)
              if ((rows >> (k * T::CPR)) & ((1ull << T::CPR) - 1)) bad |= 1ull << (i * T::RPI + k);
          }
          poison |= sees<T::NKB>(s, bad, hh);
        }
        asm volatile("" ::: "memory");
      }
      mfma_stream<T, true, 0, 0, kPrefetch>(smem, va, ka, pb, qf, o, s);
      r.l += row_sum<T>(pb);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V has been read
      if (next < n_blocks) load_rows(IC<0>{}, vbase, p.v_stride_b, next * F::KEYS, vbuf);
      block = next;
      turn ^= 1;
    }
    poison = either_half(poison);
    if (__builtin_amdgcn_ballot_w64(poison) != 0) {
      int doc;
      const int klim = row_mask(doc);
      add_not_finite<T>(p, vbase, kdoc, first_block * F::KEYS, n_blocks * F::KEYS < lim ? n_blocks * F::KEYS : lim, F::KEYS, F::KEYS * F::WAVES, klim, doc, hh, poison, o);
    }
  }

  // The results, unnormalised, through the wavefronts' own buffers: 16-byte chunk j of column i at j ^ i.
  constexpr int CH = D / 4;
#pragma unroll
  for (int db = 0; db < T::NDB; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int ch = 8 * db + 2 * g + hh;
      const f32x4 f = {o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
      *(lds_u32x4*)(uintptr_t)(kbuf + (uint32_t)(L.l32 * (D * 4) + ((ch ^ (L.l32 & (CH - 1))) * 16))) = __builtin_bit_cast(u32x4, f);
    }
  typedef __attribute__((address_space(3))) float lds_f32;
  const uint32_t state = lds + F::STATE_OFF;
  const float l = r.l + __shfl_xor(r.l, 32), lx = r.lx + __shfl_xor(r.lx, 32);
  if (hh == 0) {
    *(lds_f32*)(uintptr_t)(state + (uint32_t)(wave * 32 + L.l32) * 4u) = l > 0.f || l != l ? r.m_ref * c : -__builtin_inff();
    *(lds_f32*)(uintptr_t)(state + (uint32_t)(F::WAVES * 32 + wave * 32 + L.l32) * 4u) = l;
    *(lds_f32*)(uintptr_t)(state + (uint32_t)(2 * F::WAVES * 32 + wave * 32 + L.l32) * 4u) = lx;
  }
  wg_barrier();
  for (int e = tid; e < n_cols * CH; e += 64 * F::WAVES) {
    const int cc = e / CH, ch = e % CH;
    float m[F::WAVES], top = -__builtin_inff(), sum = 0.f, sumx = 0.f;
#pragma unroll
    for (int i = 0; i < F::WAVES; ++i) {
      m[i] = *(lds_f32*)(uintptr_t)(state + (uint32_t)(i * 32 + cc) * 4u);
      top = __builtin_fmaxf(top, m[i]);
    }
    if (top == -__builtin_inff()) top = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < F::WAVES; ++i) {
      const float w = __builtin_amdgcn_exp2f(m[i] - top);
      sum = __builtin_fmaf(w, *(lds_f32*)(uintptr_t)(state + (uint32_t)((F::WAVES + i) * 32 + cc) * 4u), sum);
      sumx = __builtin_fmaf(w, *(lds_f32*)(uintptr_t)(state + (uint32_t)((2 * F::WAVES + i) * 32 + cc) * 4u), sumx);
      const f32x4 f = __builtin_bit_cast(f32x4, *(lds_u32x4*)(uintptr_t)(lds + (uint32_t)(i * F::WAVE_B + cc * (D * 4) + ((ch ^ (cc & (CH - 1))) * 16))));
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] = __builtin_fmaf(w, f[k], acc[k]);
    }
    const bool any = sum > 0.f || sum != sum;
    const float inv = any ? 1.f / sum : 0.f;
    const int rr = cc / group, hd = kv_head * group + (cc - rr * group);
    const int64_t rh = (int64_t)(sq.q_start + rr) * n_heads + hd;
    const float row_lse = any ? kLn2 * (top + __builtin_amdgcn_logf(sumx)) : -__builtin_inff();
    if (sq.parts > 1) {
      const int64_t prh = (sq.part_row + (int64_t)part * lq + rr) * n_heads + hd;
      const f32x4 y = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
      store_through(reinterpret_cast<u32x4*>(p.part_out + prh * D + ch * 4), __builtin_bit_cast(u32x4, y));
      if (ch == 0) p.part_lse[prh] = row_lse;
    } else {
      const u32x2 y = {pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
      *reinterpret_cast<u32x2*>(static_cast<char*>(p.out) + rh * (2 * D) + ch * 8) = y;
      if (ch == 0 && p.lse != nullptr) p.lse[rh] = row_lse;
    }
  }
#endif
}

// ---------------------------------------------------------------------------------------------
// out = sum over parts exp(lse_part - lse) O_part.  A wavefront for a (row, head): a lane holds the weight of a part, then two
// elements (D 64: one) of the row.  Two latencies, of the parts' lse and of the parts themselves.  Eight rows x 24 heads in up to 17
// parts 4.9 us (one thread for eight elements, which goes through the parts: 8.2), 226 x 24 in ten parts 7.5.
// ---------------------------------------------------------------------------------------------
constexpr int kJoinRows = 4;  // (row, head)s of a workgroup

template <int D>
__global__ void __launch_bounds__(256) masked_join_kernel(MaskedParams p, int32_t n) {
  typedef __attribute__((__vector_size__(D / 64 * sizeof(float)))) float elems;
  const MaskedSeq& sq = find_seq<&MaskedSeq::join0>(p, n, blockIdx.x);
  const int lane = threadIdx.x & 63, parts = sq.parts;
  const int64_t rh = (int64_t)(blockIdx.x - sq.join0) * kJoinRows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n_rh = (int64_t)sq.q_len * p.n_heads;
  if (rh >= n_rh) return;
  const int64_t rh0 = sq.part_row * p.n_heads + rh;
  static_assert(kMaskedMaxParts == 64, "a lane for each part");
  const float part_lse = lane < parts ? p.part_lse[rh0 + lane * n_rh] : -__builtin_inff();
  const float* src = p.part_out + rh0 * D + lane * (D / 64);
  float top = part_lse;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, d));
  if (top == -__builtin_inff()) top = 0.f;
  const float w = __builtin_amdgcn_exp2f((part_lse - top) * 1.44269504088896340736f);
  float sum = w;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  elems acc = {};
  auto add = [&](elems x, int i) {
    const float wi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i));
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
      // A weight that is 0 in 32 bits keeps what is not finite, as in a call without parts.  (Nothing seen: x is 0.)
      const bool keep = wi == 0.f && !(__builtin_fabsf(x[k]) < __builtin_inff());
      acc[k] = keep ? acc[k] + x[k] : __builtin_fmaf(wi, x[k], acc[k]);
    }
  };
  int i = 0;
  for (; i + 8 <= parts; i += 8) {
    elems x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const elems*>(src + (i + j) * n_rh * D);
#pragma unroll
    for (int j = 0; j < 8; ++j) add(x[j], i + j);
  }
  for (; i < parts; ++i) add(*reinterpret_cast<const elems*>(src + i * n_rh * D), i);
  const bool any = sum > 0.f || sum != sum;
  const float inv = any ? 1.f / sum : 0.f;
  const int64_t to = (int64_t)sq.q_start * p.n_heads + rh;
  if constexpr (D == 128) {
    static_cast<uint32_t*>(p.out)[to * 64 + lane] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  } else {
    static_cast<__bf16*>(p.out)[to * 64 + lane] = (__bf16)(acc[0] * inv);
  }
  if (p.lse != nullptr && lane == 0) p.lse[to] = any ? top + kLn2 * __builtin_amdgcn_logf(sum) : -__builtin_inff();
}

// ---------------------------------------------------------------------------------------------
// Launch
// ---------------------------------------------------------------------------------------------
using MaskedKernel = void (*)(MaskedParams);
struct MaskedEntry {
  MaskedKernel fn;
  int lds, threads;
};

template <int D, bool CAP, bool BIAS>
static MaskedEntry entry_of(bool few_rows, bool lse) {
  using T = Tile<D, 4, 64>;
  if (few_rows) return {masked_few_rows_kernel<D, CAP, BIAS>, FewRows<D>::LDS_BYTES, 64 * FewRows<D>::WAVES};
  if (lse) return {masked_attn_kernel<T, CAP, BIAS, true>, kMaskedLds<T>, T::NT};
  return {masked_attn_kernel<T, CAP, BIAS, false>, kMaskedLds<T>, T::NT};
}
template <int D>
static MaskedEntry entry_of(const MaskedKind& k) {
  if (k.cap) return k.bias ? entry_of<D, true, true>(k.few_rows, k.lse) : entry_of<D, true, false>(k.few_rows, k.lse);
  return k.bias ? entry_of<D, false, true>(k.few_rows, k.lse) : entry_of<D, false, false>(k.few_rows, k.lse);
}
static MaskedEntry entry_of(const MaskedKind& k) { return k.head_dim == 64 ? entry_of<64>(k) : entry_of<128>(k); }

hipError_t masked_attn_prepare() {
  for (int i = 0; i < 32; ++i) {
    const MaskedKind k = {i & 1 ? 128 : 64, (i & 2) != 0, (i & 4) != 0, (i & 8) != 0, (i & 16) != 0};
    const MaskedEntry m = entry_of(k);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(m.fn), hipFuncAttributeMaxDynamicSharedMemorySize, m.lds);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t masked_attn_launch(const MaskedParams& p, const MaskedKind& kind, uint32_t n_doc_tiles, hipStream_t stream) {
  if (p.n_items == 0) return hipSuccess;
  if (n_doc_tiles > 0) {
    hipLaunchKernelGGL(masked_doc_tiles_kernel, dim3((n_doc_tiles + 3) / 4), dim3(256), 0, stream, p, n_doc_tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const MaskedEntry m = entry_of(kind);
  hipLaunchKernelGGL(m.fn, dim3(p.n_items), dim3(m.threads), m.lds, stream, p);
  return hipGetLastError();
}

uint32_t masked_join_blocks(const MaskedSeq& s, int n_heads) {
  return (uint32_t)(((int64_t)s.q_len * n_heads + kJoinRows - 1) / kJoinRows);
}

hipError_t masked_join_launch(const MaskedParams& p, int32_t n, uint32_t n_blocks, int head_dim, hipStream_t stream) {
  if (n == 0) return hipSuccess;
  const auto fn = head_dim == 64 ? masked_join_kernel<64> : masked_join_kernel<128>;
  hipLaunchKernelGGL(fn, dim3(n_blocks), dim3(256), 0, stream, p, n);
  return hipGetLastError();
}

}  // namespace dit
