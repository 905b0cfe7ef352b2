// What the two decode kernels (bf16 caches: decode.hip, 4-bit caches: decode_q4.hip) share: the parameters of a launch, the
// query's row of the pattern in closed form, the packets with which workgroups merge, the layout of partial outputs in LDS.
#pragma once
#include "common.h"

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int CH = 64;         // tokens per chunk
constexpr int NW = 8;          // wavefronts per workgroup
constexpr int MAXG = 16;       // query heads per KV head (columns of the MFMA tile)

struct dec_params {
  const __bf16* q; const __bf16* k; const __bf16* v; const int32_t* kv_len;
  __bf16* o; float* lse;
  float* partials;      // [batch, hq, splits, D + 2] floats when splits > 1 and a merge kernel follows
  uint64_t* packets;    // the same shape as (value, tag) packets when the workgroups merge among themselves
  uint32_t* gen;        // [batch, hkv] generation numbers of the packets (any initial value)
  int64_t capacity;
  int32_t len_max;      // the capacity, or the largest sequence length that there is
  int32_t B, W, S; uint32_t flags;
  int32_t hq, hkv, G, splits, subs;
  uint32_t subs_magic;  // ceil(2^32 / subs) for subs > 1: slot / subs = umulhi(slot, subs_magic) for every slot of a row
  uint32_t per_b_magic; // persistent workgroups: ceil(2^32 / items of a sequence) where that replaces the division of any item's number (else 0)
  int32_t kvh_first;    // 1: the KV head is the fastest digit of a workgroup's number, 0: the split
  int32_t through;      // 1: packets are taken back with stores that go through to memory
  int32_t fused;        // 1: the workgroups of a (sequence, KV head) merge their partials among themselves
  float c2;
  const int32_t* block_table;   // paged cache: page of block j of sequence b at [b * table_stride + j]; else null
  int32_t table_stride;
  int32_t last_page;            // the pool's last page (that an entry of the table can name)
};

// ---- merging the workgroups of a (sequence, KV head) without a second kernel ----
// Every value of a partial result travels as one 8-byte packet (value, tag), written and read with single 8-byte
// device-scope accesses, so a reader sees a value together with its tag or not at all.  The tag is derived from the
// generation number g that the (sequence, KV head) keeps in the workspace, read at the start of the kernel, and from
// the split.  Protocol of a workgroup: store its packets; wait until memory has acknowledged every one of them
// (s_waitcnt, then the workgroup's barrier); load the packets of the other splits; if every tag is the expected one,
// combine all partials in split order, write the output and store g + 1 as the new generation.
//  * Some workgroup finishes: order the workgroups by the time at which the last of their stores was acknowledged;
//    the latest one loads after that, when every other workgroup's packets are in memory.
//  * Several may finish: they combine the same values in the same order and write the same bits.  (Each thread decides for
//    the outputs it owns: a vote of the workgroup took another 0.6 us.)
//  * Nothing stale is taken for valid.  An output's packet is taken back by the thread that used it (its tag becomes 0, and
//    a valid one is odd): no call leaves one behind, whatever the memory is used for before it is a workspace again, its
//    words g put back to old ones included, and also where a graph replays the launch.  Maxima and sums are shared by the
//    threads of a head and stay; those of the call before carry generation g - 1 (the finisher advanced it only after every
//    workgroup of the pair had stored packets, hence all of its wavefronts had read g, before the barrier in front of its
//    stores), and older ones whose generation is back do not fit the output's packet, whose tag is formed with the bits of
//    the maximum and the sum that go with it.  The very first call on a workspace meets whatever the memory held: a word
//    there passes for the tag of a maximum only if it equals ~g ^ ((split + 1) << 24) for the word g found in the same
//    memory (never for a memory filled with one byte value, zeros included).
//  * No workgroup waits for another one: whoever finds a packet missing simply leaves.  (A look before the acknowledgement
//    may find everything in place already; only the one after it has to be there.)
// Calls that may run at the same time must not share a workspace (they would share generation numbers).
// With more splits than this a merge kernel follows: what a workgroup reads grows with their number.  us, merged among
// themselves / by the kernel, 32 query heads on 8: 7 splits, batch 2 10.35 / 8.9, 5 19.8 / 15.2 (batch 1 level); 8 splits, batch 4,
// 29 chunks 12.3 / 10.9, 62 chunks 18.2 / 15.7, batch 8 37.8 / 32.5, 128 heads on 8 24.2 / 13.5.  Up to 6 the kernel's time on the
// GPU is no longer either (6 splits, batch 1 8.7 / 7.85), but its launch takes the host longer than the step takes the GPU:
// launched from Python, one after another, such steps were paced at 8.7 to 9.1 us on some hosts.
constexpr int MAX_FUSED_SPLITS = 6;
__device__ __forceinline__ uint32_t dec_tag(uint32_t gen, int split) { return ~gen ^ ((uint32_t)(split + 1) << 24); }
// ... of an output: with the maximum and the sum of its head; odd
__device__ __forceinline__ uint32_t dec_tag_of_output(uint32_t tag, uint32_t m_bits, uint32_t l_bits) {
  return (tag ^ m_bits ^ (l_bits << 16 | l_bits >> 16)) | 1u;
}
__device__ __forceinline__ void dec_put(uint64_t* slot, float x, uint32_t tag) {
  __hip_atomic_store(slot, ((uint64_t)tag << 32) | __builtin_bit_cast(uint32_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The launch that has to see it is a later one, so an ordinary store is enough; where the launch fills the chip, it is better
// written through at once than left for the end of the kernel (us, 32 query heads on 8, not taken back / ordinary / through:
// batch 1 7.9 / 8.0 / 8.4, batch 4 9.05 / 9.05 / 9.32, batch 16 12.15 / 12.75 / 12.21; 28 on 4, ordinary: batch 2 9.4 / 9.9, 4
// 10.15 / 10.6; all of them at the end of the kernel instead: 0 to 0.5 more).
template <int SCOPE>
__device__ __forceinline__ void dec_take_back(uint64_t* first, int splits, int stride) {
#pragma unroll
  for (int y = 0; y < MAX_FUSED_SPLITS; ++y)
    if (y < splits) __hip_atomic_store(first + (int64_t)y * stride, (uint64_t)0, __ATOMIC_RELAXED, SCOPE);
}
__device__ __forceinline__ uint64_t dec_get(const uint64_t* slot) {
  return __hip_atomic_load(slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// LDS layout of the wavefronts' partial outputs: the 32 values a lane holds (d = 32*q4 + x) form a row of 36 floats,
// so that the 16 lanes of a store (4 heads x 4 groups) start 36 floats apart and cover all banks between them.
constexpr int OROW = 36;
template <int D>
__device__ __forceinline__ int dec_o_at(int wave, int G, int g, int d) { return (((wave * G + g) * (D / 32) + (d >> 5)) * OROW) + (d & 31); }
template <int D>
constexpr size_t dec_o_bytes(int G) { return (size_t)NW * G * (D / 32) * OROW * sizeof(float); }

// The query's row of the pattern in closed form: [0, sink_end) ++ {i - 2^k inside [pow_lo, win_start), k
// descending} ++ [win_start, i].  Uniform over a workgroup, so all of it runs on the scalar unit, and it stands between
// the sequence length and the first load: positions are 32-bit numbers (as the lengths are), half the instructions.
struct dec_row {
  pa_row_shape_t<int32_t> rs;
  int32_t t, i;          // position of the query, its block
  int n_pow, k_max;      // isolated blocks i - 2^k for k = k_max, k_max-1, ...: n_pow of them
  int n_slots;           // 64-token chunks of the attended blocks
};
__device__ __forceinline__ dec_row dec_row_of(const dec_params& p, int32_t len) {
  dec_row r;
  if (len < 1) len = 1;
  if (len > p.len_max) len = p.len_max;
  r.t = len - 1;
  // t / B = (t / 64) / subs: exact through the multiply-high, because t / 64 stays below 2^25
  static_assert(CH == 64, "the block index is formed from 64-token chunks");
  const unsigned chunk_of_t = (unsigned)r.t >> 6;
  r.i = p.subs == 1 ? (int)chunk_of_t : (int)__umulhi(chunk_of_t, p.subs_magic);
  r.rs = pa_shape_of_row<int32_t>(p.W, p.S, p.flags, r.i);
  const pa_row_powers pw = pa_powers_of_row<int32_t>(r.rs, p.flags, r.i);
  r.n_pow = pw.n_pow; r.k_max = pw.k_max;
  const int n_blocks = r.rs.sink_end + r.n_pow + (r.i - r.rs.win_start + 1);
  r.n_slots = n_blocks * p.subs;
  return r;
}
__device__ __forceinline__ int32_t dec_block_at(const dec_row& r, int lp) {   // lp-th attended block, ascending
  if (lp < r.rs.sink_end) return lp;
  lp -= r.rs.sink_end;
  if (lp >= r.n_pow) return r.rs.win_start + (lp - r.n_pow);
  return r.i - (1 << (r.k_max - lp));
}
// Chunk `slot` of the row: its block, the chunk inside the block, the tokens of it the query attends (<= 0: none)
struct dec_place { int32_t blk; int sub; int n_tok; };
__device__ __forceinline__ dec_place dec_place_of(const dec_params& p, const dec_row& r, int slot) {
  // (no division in the kernel: a 64-bit one costs more than the rest of the address arithmetic)
  dec_place c;
  const int lp = p.subs == 1 ? slot : (int)__umulhi((unsigned)slot, p.subs_magic);
  c.sub = slot - lp * p.subs;
  c.blk = dec_block_at(r, lp);
  const int left = (r.t - c.blk * p.B) - c.sub * CH + 1;      // causal: tokens tok0..t are attended
  c.n_tok = left >= CH ? CH : left;
  return c;
}
// First K and V row of a chunk: in the contiguous cache, or in its page (page numbers outside the pool are clamped
// into it: a bad table gives wrong numbers, never an access outside the pool)
__device__ __forceinline__ int64_t dec_chunk_offset(const dec_params& p, int b, int kvh, const dec_place& c, int page, int D) {
  if (!p.block_table) return (((int64_t)b * p.hkv + kvh) * p.capacity + (int64_t)(c.blk * p.B + c.sub * CH)) * D;
  page = page < 0 ? 0 : (page > p.last_page ? p.last_page : page);
  return (((int64_t)page * p.hkv + kvh) * p.B + c.sub * CH) * D;
}
// the table's entry for block `blk`, through the scalar unit (the table does not change while a kernel runs)
__device__ __forceinline__ int dec_page(const dec_params& p, int b, int blk) {
  typedef const __attribute__((address_space(4))) int32_t scalar_int;
  return *(scalar_int*)(uintptr_t)(p.block_table + (int64_t)b * p.table_stride + blk);
}

// A buffer of `bytes` bytes from `base` on (uniform): loads beyond its end return zeros, so the rows behind the last
// attended token and the heads behind the group's last one need no comparison, no branch and no register of their own.
typedef __amdgpu_buffer_rsrc_t dec_buf;
__device__ __forceinline__ dec_buf dec_buffer(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 dec_load16(dec_buf buf, int lane_offset, int offset) {
  return __builtin_amdgcn_raw_buffer_load_b128(buf, lane_offset + offset, 0, 0);
}
