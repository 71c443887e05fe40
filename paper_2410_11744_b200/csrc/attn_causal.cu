// Causal attention of new tokens (a chunk of a sequence over its paged cache, or whole packed prompts), for plans in which some
// request has more than 64 packed rows (tokens x GQA group); all requests of such a plan are served here, single tokens too:
//   out_i = sum_{t <= c + i} softmax_t(scale <q_i, k_t>) v_t          (token i of the chunk is token c + i of its sequence)
//
// One CTA per SM, 12 warps; a work item is 256 packed query rows of one (request, kv head), two halves A and B of 128, against
// a range of 128-key tiles:
//   warp 0       TMA producer: the item's Q (half A, then B), then K and V tiles into a shared-memory ring;
//   warps 1, 3   issue tcgen05.mma for half A / B: S = Q K^T (both operands in shared memory), O += P V (P in tensor memory);
//   warp 2       tensor memory: S_A, S_B (128 fp32 columns each), O_A, O_B (D each);
//   warps 4-7    softmax of half A, a row per thread: fp32 online softmax in the exp2 domain; warps 8-11 of half B.
// A half's P (bf16) takes the place of its S: a thread has its row of scores in registers before it writes the first
// probability.  Products of one issuing thread run in order, so S(j + 1), issued behind P V(j), overwrites a P that has
// been read, and "S(j + 1) is there" also says that P V(j) is done: one barrier tells the softmax threads both, and the
// running output may be rescaled then without another wait.
//
// What bounds it.  A tile is 2 048 cycles of the tensor pipe (D = 128, both halves), as many of the exponential unit, and about
// 1 200 issue slots of each scheduler, but its period is the chain of one half, 3 320 cycles in a trace: S to registers 180, weights
// 2 090, P V and the next S 1 050; the other half's products run beside it.  512 tokens over 8192 keys (64 / 8 heads of 128) take
// 120 - 122 us with cold inputs, 1.17 PFLOP/s (101 - 116 over and over on the same inputs, by the clock that the power cap leaves); a prompt
// of 16384 3.3 - 3.8 ms, 1.15 - 1.35 PFLOP/s, under the power cap.  What it took, each measured against the step before on those 512
// tokens (on the same inputs):
//   - Issuing in turns, A's P V and next S, then B's (153 -> 143 us).  Without turns both halves' products interleave, their S
//     arrive together, both softmaxes run at once, and then the pipe waits for them: 4 430 cycles.
//   - tcgen05.mma operands that the compiler knows to be uniform (elect.sync, values through a shuffle): 143 -> 122.  From ordinary
//     registers each product took 90 - 120 cycles to issue instead of 64.
//   - Weights against the old reference beside the maximum, not behind it; P handed over in two pieces of 64 keys, so that
//     the first half of P V runs under the second half of the weights (pieces of 32 + 96 or 96 + 32: 5 % slower).
//   - An issuer per half, so that one's waits and commits run under the other's batch (2 - 3 %).
//   - For heads of 64, 5 of 16 pairs of exponentials on the FMA pipe (see kPolyPairs).
// Tried and slower: two threads per row (16 softmax warps, 104 registers: 130 - 138); one S buffer that the halves share, with P
// beside it, as in the tree kernel (123); for D = 64, whose tensor memory has the room, P beside two S buffers (193 -> 221:
// both softmaxes at once again) or a third S buffer and an issuer that runs three products ahead, across items too (184 -> 223, the
// same); one issuer that asks for the next item's S before this one's output is out (long prompts + 3 %).
// Neither half the loads (timing only) nor a finer ring changed anything.  D = 64: 592 tokens over 15792 keys (64 / 8 heads) 202 us, cold; a
// scheduler issues in 57 % of the cycles, the exponential unit is busy in 54 %, the FMA pipe in 48, the tensor pipe in 39.
//
// An item costs about 4 us beside its tiles (a prompt of 700 tokens: a third of its time): masked tiles, the output,
// and code that runs once per item and has to be fetched again (ncu: 0.73 cycles without an instruction per instruction issued, 0.24 on
// long contexts).  Slower all the same: the next item's S in the turn of this one's last product, or without a turn (+ 3 - 20 %); the output
// read in one go (+ 3 %); masked and first tiles 32 keys at a time in a loop from tensor memory, a quarter of the code (+ 6 % even on
// long contexts: the fast path is scheduled differently); weights without a maximum, a tile's sum telling when the reference has to
// rise (7 % fewer instructions, + 5 - 10 %); half B taking every other key tile of an item that has rows for half A only (batches of single
// tokens with heads of 64 - 18 %, everything with two halves + 4 - 8 %).
//
// CTAs take items from a queue, longest first (see schedule_causal in api.cu); an item whose group was cut along the
// keys writes an fp32 partial (O, m, l) that combine_kernel merges.  Every wait on an mbarrier is bounded (see mbar_wait_idle).
#include "tc_ops.cuh"
#include <type_traits>

namespace dyspec {

namespace {

constexpr int BMH = 128;          // rows of one query half
constexpr int BN = 128;           // keys per tile
constexpr int kThreads = 384;
constexpr uint32_t kTmemCols = 512;
constexpr float kRescaleThreshold = 8.0f;   // log2 units: the output is rescaled only when a row maximum grows by more

template <int D>
struct CausalLayout {
  static constexpr int kSlots = D == 128 ? 5 : 10;            // K / V tiles in the ring
  static constexpr int kPanels = D / 64;
  static constexpr int kPanelBytes = 128 * 128;               // 128 rows x 128 bytes
  static constexpr int kTileBytes = kPanels * kPanelBytes;    // one K tile, V tile or query half
  static constexpr int kRingOffset = 2 * kTileBytes;
  static constexpr int kBarOffset = kRingOffset + kSlots * kTileBytes;
  static constexpr int kItemRingOffset = kBarOffset + 512;    // the CTA's next work items, 8 entries of 64 bytes
  static constexpr int kTotal = kItemRingOffset + 512;
};

// mbarriers (8 bytes each), behind them: tensor-memory address, abort flag, indexes of the item ring
template <int kSlots>
struct Bars {
  static constexpr int kQFull = 0;                      // [2] query half A / B is in shared memory
  static constexpr int kQFree = 2;                      // the item's last S products have run
  static constexpr int kSlotFull = 3;                   // [kSlots]
  static constexpr int kSlotEmpty = kSlotFull + kSlots; // [kSlots] two commits, one per issuer
  static constexpr int kSReady = kSlotEmpty + kSlots;   // [2]
  static constexpr int kODone = kSReady + 2;            // [2] the item's last P V has run
  static constexpr int kOFree = kODone + 2;             // [2] the output has been read out
  static constexpr int kItemFull = kOFree + 2;          // [8] item ring entry written
  static constexpr int kItemEmpty = kItemFull + 8;      // [8] ... and read by the issuing and softmax warps
  static constexpr int kCount = kItemEmpty + 8;
};

// 2^x for x <= 127 on the FMA pipe, two at a time: x = n + f with n the nearest integer, 2^f by the quintic through 1 at f = 0 with the
// smallest largest relative error on [-1/2, 1/2] (found as a linear program; 1.6e-7 as evaluated in fp32, the 2^-22 that the
// exponential unit is held to is 2.4e-7), n added to its exponent.  Below -125 the result stays at 2^-125 (relative to a row's
// largest term of 1, nothing); a NaN is the caller's to keep away.
__device__ __forceinline__ uint64_t exp2_poly2(uint64_t x2) {
  constexpr float kMagic = 12582912.f;      // 1.5 * 2^23: adding it leaves the nearest integer in the low bits
  float x0, x1, t0, t1, p0, p1;
  unpack_f32x2(x2, x0, x1);
  x2 = pack_f32x2(fmaxf(x0, -125.f), fmaxf(x1, -125.f));
  const uint64_t t2 = add_f32x2(x2, pack_f32x2(kMagic, kMagic));
  const uint64_t n2 = add_f32x2(t2, pack_f32x2(-kMagic, -kMagic));
  const uint64_t f2 = fma_f32x2(n2, pack_f32x2(-1.f, -1.f), x2);
  auto both = [](float c) { return pack_f32x2(c, c); };
  uint64_t p2 = fma_f32x2(both(0.00132647273f), f2, both(0.00967151299f));
  p2 = fma_f32x2(p2, f2, both(0.0555073358f));
  p2 = fma_f32x2(p2, f2, both(0.240222424f));
  p2 = fma_f32x2(p2, f2, both(0.693147004f));
  p2 = fma_f32x2(p2, f2, both(1.f));
  unpack_f32x2(t2, t0, t1);
  unpack_f32x2(p2, p0, p1);
  return pack_f32x2(__uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23)),
                    __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23)));
}
// Of the 16 pairs in 32 keys, how many take the polynomial.  Heads of 128 have products twice as long to hide the exponential unit under:
// none (512 tokens over 8192 keys, 64 / 8 heads, call after call: 121.4 us, 2 - 5 pairs 122.6 - 123.7; one call on an idle card, at the full
// clock: 136.7, 4 pairs 134.2).  Heads of 64 (592 tokens over 15792 keys, 64 / 8 heads): 202 us with 5 pairs, 208 - 214 with 0, 4, 6 or 7.
// (A cubic, 7.5e-5, would give 196, and heads of 128 131.5 on an idle card: not worth bits that the header promises.)
template <int D>
constexpr int kPolyPairs = D == 128 ? 0 : 5;
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// Trace tags (see dyspec_set_trace): role << 14 | event << 10 | key-tile index; roles 0 / 3 = issuer of half A / B, 1 / 2 = softmax row 0
// of half A / B.  Issuer events: 1 / 3 first / second 64 keys of P seen, 2 turn taken, 4 products issued.  Softmax events: 1 S seen, 2
// row loaded, 3 maximum known, 4 / 5 first / second 64 keys of P published, 6 last P V seen, 7 output written.
#define DYSPEC_TAG(role, event, j) ((uint32_t(role) << 14) | (uint32_t(event) << 10) | (uint32_t(j) & 1023u))

// One lane of the warp, and the compiler knows that it is one: what feeds a tcgen05 instruction stays in uniform registers.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one) :: "memory");
  return one != 0;
}


constexpr int kFirstChunks = 2;          // P is handed over in two pieces: 32 * kFirstChunks keys, then the rest
constexpr int kBarP = 1;                    // named barriers 1 .. 4: 64 keys of P are in tensor memory (half A: 1, 2; half B: 3, 4)
constexpr int kBarTurn = 5;                 // named barriers 5, 6: half A's / half B's turn to issue
constexpr int kPCount = BMH + 32;           // a half's softmax threads + the issuing warp

}  // namespace

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
causal_attn_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const AttnParams p, const __grid_constant__ FirstItems first) {
  using L = CausalLayout<D>;
  constexpr int kSlots = L::kSlots;
  using Br = Bars<kSlots>;
  static_assert(8 * Br::kCount + 48 <= 512, "barrier area");
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t s_q = smem_u32(smem);
  const uint32_t s_ring = s_q + L::kRingOffset;
  const uint32_t s_bar = s_q + L::kBarOffset;
  auto bar = [&](int i) { return s_bar + 8u * uint32_t(i); };
  volatile uint32_t* tmem_holder = reinterpret_cast<volatile uint32_t*>(smem + L::kBarOffset + 8 * Br::kCount);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kBarOffset + 8 * Br::kCount + 8);
  volatile int32_t* ring_idx = reinterpret_cast<volatile int32_t*>(smem + L::kBarOffset + 8 * Br::kCount + 16);
  uint4* ring_item = reinterpret_cast<uint4*>(smem + L::kItemRingOffset);

  const int warp = __shfl_sync(0xffffffffu, int(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int h = 0; h < 2; ++h) {
      mbar_init(bar(Br::kQFull + h), 1);
      mbar_init(bar(Br::kSReady + h), 1);
      mbar_init(bar(Br::kODone + h), 1);
      mbar_init(bar(Br::kOFree + h), BMH);
    }
    mbar_init(bar(Br::kQFree), 2);
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(bar(Br::kSlotFull + s), 1);
      mbar_init(bar(Br::kSlotEmpty + s), 2);
    }
    for (int e = 0; e < 8; ++e) {
      mbar_init(bar(Br::kItemFull + e), 1);
      mbar_init(bar(Br::kItemEmpty + e), 2 + 2 * BMH / 32);
    }
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(const_cast<uint32_t*>(tmem_holder))), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_holder, 0);

  // The CTA's first item is item blockIdx.x of the queue and travels with the kernel parameters; the producer warp takes
  // further ones with an atomic add and passes them on through a ring of 8 entries.  No queue (p.queue null): one item per CTA.
  const bool first_here = blockIdx.x < kFirstItems;
  auto item_of = [&](int w, bool consumer = true) -> WorkItem {
    if (w == 0) return first_here ? first.item[blockIdx.x] : p.items[blockIdx.x];
    union { WorkItem it; uint4 v[4]; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.v[i] = ring_item[((w - 1) & 7) * 4 + i];
    if (consumer) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Br::kItemEmpty + ((w - 1) & 7)));
    }
    return u.it;
  };
  auto take_item = [&](int w) -> bool {                    // producer warp, all lanes
    if (w == 0) return true;
    if (p.queue == nullptr) return false;
    int idx = 0;
    if (lane == 0) {
      if (w == 1) grid_dependency_wait();                  // the last launch on this workspace cleared the queue words
      const int t = atomicAdd(p.queue, 1) + int(gridDim.x);
      if (w > 8) mbar_wait_idle(bar(Br::kItemEmpty + ((w - 1) & 7)), (uint32_t((w - 1) >> 3) & 1u) ^ 1u, abort_flag, p.status);
      idx = t < p.n_items_total ? t : -1;
      ring_idx[(w - 1) & 7] = idx;
      if (idx >= 0) {
        const uint4* src = reinterpret_cast<const uint4*>(p.items + idx);
#pragma unroll
        for (int i = 0; i < 4; ++i) ring_item[((w - 1) & 7) * 4 + i] = __ldg(src + i);
      }
      mbar_arrive(bar(Br::kItemFull + ((w - 1) & 7)));     // (release: the entry is written)
      if (idx < 0 && atomicAdd(p.queue + 1, 1) == int(gridDim.x) - 1) {   // every CTA has found the queue empty
        p.queue[0] = 0;
        p.queue[1] = 0;
      }
    }
    __syncwarp();
    return __shfl_sync(0xffffffffu, idx, 0) >= 0;
  };
  auto next_item = [&](int w) -> bool {                    // the other roles
    if (w == 0) return true;
    if (p.queue == nullptr) return false;
    // The producer publishes every item in bounded time, whatever other waits ran out: a role that is in its error state still
    // goes through the items that the others go through, so that all of them meet at the named barriers.
    const uint32_t at = bar(Br::kItemFull + ((w - 1) & 7)), parity = uint32_t((w - 1) >> 3) & 1u;
    if (!mbar_wait_idle(at, parity, abort_flag, p.status)) {
      const uint64_t t0 = global_timer_ns();
      while (!mbar_test_wait(at, parity))
        if (global_timer_ns() - t0 > 8 * kWaitLimitNs) return false;
    }
    return ring_idx[(w - 1) & 7] >= 0;
  };
  const int g = p.group_size;
  auto halves = [&](const WorkItem& it) { return it.n_nodes * g - it.row0 > BMH ? 2 : 1; };
  // Key tiles of an item that half h takes part in: half A's rows may see nothing of the last one of an item with both halves
  // (its 128 rows are at most 128 tokens, so all others concern both).
  auto half_tiles = [&](const WorkItem& it, int h) {
    const int T = it.tile_end - it.tile_begin;
    const int last_key = it.prefix_len + ((it.row0 + BMH - 1) >> p.log2_g);          // of half A
    return T - (h == 0 && T > 1 && halves(it) == 2 && last_key < (it.tile_end - 1) * BN ? 1 : 0);
  };

  trigger_dependents();     // the next kernel of the stream may be scheduled; it waits for this grid before it touches what this one writes
  if (warp < 4) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (one lane issues)
    const bool elected = lane == 0;
    if (elected) {
      prefetch_tensormap(&map_q);
      prefetch_tensormap(&map_k);
      prefetch_tensormap(&map_v);
    }
    uint32_t slot = 0, ph = 0;
    for (int w = 0; take_item(w); ++w) {
      const WorkItem item = item_of(w, false);
      const int nh = halves(item);
      mbar_wait_idle(bar(Br::kQFree), (uint32_t(w) & 1u) ^ 1u, abort_flag, p.status);
      // half A, the first K tile, half B: the item's first product needs only the first two
      auto load_q_half = [&](int h) {
        if (elected) {
          mbar_expect_tx(bar(Br::kQFull + h), L::kTileBytes);
          for (int pn = 0; pn < L::kPanels; ++pn)
            tma_load_3d(s_q + h * L::kTileBytes + pn * L::kPanelBytes, &map_q, bar(Br::kQFull + h), pn * 64, item.kv_head * g,
                        item.node0 + ((item.row0 + h * BMH) >> p.log2_g));
        }
      };
      load_q_half(0);
      for (int t = item.tile_begin; t < item.tile_end; ++t) {
        const int64_t row = causal_tile_row(p, item, t, BN);
        for (int kv = 0; kv < 2; ++kv) {
          mbar_wait_idle(bar(Br::kSlotEmpty + slot), ph ^ 1u, abort_flag, p.status);
          if (elected) {
            mbar_expect_tx(bar(Br::kSlotFull + slot), L::kTileBytes);
            for (int pn = 0; pn < L::kPanels; ++pn)
              tma_load_3d(s_ring + slot * L::kTileBytes + pn * L::kPanelBytes, kv == 0 ? &map_k : &map_v,
                          bar(Br::kSlotFull + slot), pn * 64, item.kv_head, int(row));
          }
          if (++slot == kSlots) { slot = 0; ph ^= 1u; }
          if (t == item.tile_begin && kv == 0 && nh == 2) load_q_half(1);
        }
      }
    }
  } else if (warp == 1 || warp == 3) {
    // ------------------------------------------------------------------ tcgen05.mma issuers of half A / B (one lane issues)
    // Batch by batch in turn: A's P V and next S, B's P V and next S, ...; the turn passes through a named barrier.
    const int h = warp == 1 ? 0 : 1;
    const bool elected = lane == 0;
    TraceCursor trace = trace_open(p, h == 0 ? 0 : 3, 4);
    if (!elected) trace.at = nullptr;
    constexpr uint32_t idesc_qk = make_idesc(BN, 0);
    constexpr uint32_t idesc_pv = make_idesc(D, 1);
    constexpr uint32_t kHi = desc_hi(1024);               // 8-row (8-key) groups 1024 bytes apart
    const uint32_t q_lo = desc_lo(s_q, 16) + uint32_t(h) * (L::kTileBytes >> 4);
    const uint32_t ring_k_lo0 = desc_lo(s_ring, 16);
    const uint32_t ring_v_lo0 = desc_lo(s_ring, L::kPanelBytes);   // MN-major: leading offset = next 64-column panel
    const uint32_t t_s = tmem_base + uint32_t(h) * 128u, t_o = tmem_base + 256u + uint32_t(h) * 128u;
    auto issue_qk = [=](uint32_t slot) {
      const uint32_t b_lo = ring_k_lo0 + __shfl_sync(0xffffffffu, slot, 0) * (L::kTileBytes >> 4);
      if (elect_one()) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint32_t off = (uint32_t(ks >> 2) * L::kPanelBytes + uint32_t(ks & 3) * 32u) >> 4;
          umma_ss_lohi(t_s, q_lo + off, kHi, b_lo + off, kHi, idesc_qk, ks > 0 ? 1u : 0u);
        }
      }
      __syncwarp();
    };
    auto issue_pv = [=](uint32_t slot, auto piece_tag, bool accumulate) {
      constexpr int kFrom = decltype(piece_tag)::value ? 2 * kFirstChunks : 0, kTo = decltype(piece_tag)::value ? BN / 16 : 2 * kFirstChunks;
      const uint32_t b_lo = ring_v_lo0 + __shfl_sync(0xffffffffu, slot, 0) * (L::kTileBytes >> 4);
      if (elect_one()) {
#pragma unroll
        for (int kk = kFrom; kk < kTo; ++kk) {
          umma_ts_lohi(t_o, t_s + uint32_t(kk) * 8u, b_lo + uint32_t(kk) * (2048u >> 4), kHi, idesc_pv,
                       (accumulate || kk > kFrom) ? 1u : 0u);
        }
      }
      __syncwarp();
    };
    uint32_t slot = 0, ph = 0;                            // ring position
    uint32_t n_it = 0;                                    // items this half took part in
    bool owed = false;                                    // half A: half B's last batch has not been waited for
    for (int w = 0; next_item(w); ++w) {
      const WorkItem item = item_of(w);
      const bool two = __shfl_sync(0xffffffffu, halves(item), 0) == 2;
      const int T = __shfl_sync(0xffffffffu, item.tile_end - item.tile_begin, 0);
      const int T_h = __shfl_sync(0xffffffffu, half_tiles(item, h), 0);
      if (h == 1 && !two) {                               // no rows for this half: step over the item's tiles
        slot += 2u * uint32_t(T);
        ph ^= (slot / kSlots) & 1u;
        slot %= kSlots;
        continue;
      }
      auto take_turn = [&]() {
        if (!two) return;
        __syncwarp();
        if (h == 1 || owed) named_sync(kBarTurn + h, 64);
        owed = true;
      };
      auto pass_turn = [&]() {
        __syncwarp();
        if (two) named_arrive(kBarTurn + 1 - h, 64);
      };
      // one of the two commits that free a slot / the Q tile (half A gives both where it is alone)
      auto release = [&](int b) {
        if (elect_one()) {
          tc_commit(bar(b));
          if (!two) tc_commit(bar(b));
        }
      };
      mbar_wait_idle(bar(Br::kQFull + h), (h == 0 ? uint32_t(w) : n_it) & 1u, abort_flag, p.status);
      mbar_wait_idle(bar(Br::kSlotFull + slot), ph, abort_flag, p.status);
      take_turn();
      tc_fence_after();
      issue_qk(slot);
      if (elect_one()) tc_commit(bar(Br::kSReady + h));
      pass_turn();
      release(Br::kSlotEmpty + slot);
      if (T == 1) release(Br::kQFree);
      if (++slot == kSlots) { slot = 0; ph ^= 1u; }
      // A tile: O += P V in two pieces, behind it the next S (all tiles but the half's last)
      auto tile = [&](int j, auto more_tag) {
        constexpr bool kMore = decltype(more_tag)::value;
        const uint32_t vslot = slot, vph = ph;
        if (++slot == kSlots) { slot = 0; ph ^= 1u; }
        const uint32_t kslot = slot, kph = ph;
        if (kMore && ++slot == kSlots) { slot = 0; ph ^= 1u; }
        const uint32_t got = kMore ? mbar_test_wait2(bar(Br::kSlotFull + vslot), vph, bar(Br::kSlotFull + kslot), kph) : 2u;
        if (!(got & 1u)) mbar_wait_idle(bar(Br::kSlotFull + vslot), vph, abort_flag, p.status);
        if (!(got & 2u)) mbar_wait_idle(bar(Br::kSlotFull + kslot), kph, abort_flag, p.status);
        if (j == 0) mbar_wait_idle(bar(Br::kOFree + h), (n_it & 1u) ^ 1u, abort_flag, p.status);
        __syncwarp();
        named_sync(kBarP + 2 * h, kPCount);
        trace_event(trace, DYSPEC_TAG(3 * h, 1, j));
        take_turn();
        tc_fence_after();
        trace_event(trace, DYSPEC_TAG(3 * h, 2, j));
        issue_pv(vslot, std::integral_constant<int, 0>{}, j > 0);
        __syncwarp();
        named_sync(kBarP + 2 * h + 1, kPCount);
        tc_fence_after();
        trace_event(trace, DYSPEC_TAG(3 * h, 3, j));
        issue_pv(vslot, std::integral_constant<int, 1>{}, true);
        if constexpr (kMore) issue_qk(kslot);
        if (elect_one()) tc_commit(bar((kMore ? Br::kSReady : Br::kODone) + h));
        trace_event(trace, DYSPEC_TAG(3 * h, 4, j));
        pass_turn();
        release(Br::kSlotEmpty + vslot);
        if constexpr (kMore) release(Br::kSlotEmpty + kslot);
      };
#pragma unroll 1
      for (int j = 0; j + 1 < T_h; ++j) tile(j, std::true_type{});
      if (T_h == T && T > 1) release(Br::kQFree);         // (the last S product of this half has been issued)
      tile(T_h - 1, std::false_type{});
      if (T_h < T) {                                      // half A steps over the item's last K and V tile
        release(Br::kQFree);
        take_turn();
        pass_turn();
        for (int kv = 0; kv < 2; ++kv) {                  // (released once they are there: the slot's earlier use is over then)
          mbar_wait_idle(bar(Br::kSlotFull + slot), ph, abort_flag, p.status);
          __syncwarp();
          release(Br::kSlotEmpty + slot);
          if (++slot == kSlots) { slot = 0; ph ^= 1u; }
        }
      }
      ++n_it;
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ------------------------------------------------------------------ softmax + epilogue warps
    // The work items are written before the launch; Q, K, V and the page table are inputs that the kernels in front do not write when
    // they signal early launch (no attention output without an ordinary kernel in between: the header's rule on stream
    // order).  Only the output and the partials wait for the preceding kernels of the stream.
    bool dep_ok = false;
    const int h = (warp - 4) >> 2;                       // query half
    const int r = ((warp & 3) << 5) + lane;              // row of the half == TMEM lane
    const uint32_t lane_sel = uint32_t((warp & 3) << 5) << 16;
    const uint32_t t_s = tmem_base + uint32_t(h) * 128u + lane_sel;             // scores, then probabilities (bf16 pairs)
    const uint32_t t_o = tmem_base + 256u + uint32_t(h) * 128u + lane_sel;
    uint32_t n_s = 0, n_o = 0;                           // S-ready / O-done phases seen
    uint32_t ring = 0;                                   // K and V tiles of earlier items
    TraceCursor trace = trace_open(p, 1 + h, 4);
    if (r != 0) trace.at = nullptr;

    for (int w = 0; next_item(w); ++w) {
      const WorkItem item = item_of(w);
      const int n_rows = item.n_nodes * g;
      const uint32_t ring0 = ring;                                  // K tile j at ring position ring0 + 2 j, its V tile behind it
      ring += 2u * uint32_t(item.tile_end - item.tile_begin);
      if (h >= halves(item)) continue;
      const int T = half_tiles(item, h);
      const int row = item.row0 + h * BMH + r;
      const bool ok = row < n_rows;
      const int token = min(row >> p.log2_g, item.n_nodes - 1);     // (rows behind the last one follow it; they are not written)
      const int last_key = item.prefix_len + token;                 // the row sees keys 0 .. last_key

      float m_used = -INFINITY, l = 0.f;
      for (int j = 0; j < T; ++j) {
        const int key0 = (item.tile_begin + j) * BN;
        const int vis = last_key + 1 - key0;                        // how many of the tile's keys the row sees (<= 0: none, >= 128: all)
        const bool all_visible = __all_sync(0xffffffffu, vis >= BN);
        const int own = item.prefix_len + item.n_nodes - key0;      // how many of them belong to the sequence
        mbar_wait_idle(bar(Br::kSReady + h), n_s & 1u, abort_flag, p.status);
        ++n_s;
        __syncwarp();
        tc_fence_after();
        trace_event(trace, DYSPEC_TAG(1 + h, 1, j));
        uint32_t sv[BN];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(t_s + uint32_t(c) * 32u, sv + 32 * c);
        tmem_wait_ld();
        trace_event(trace, DYSPEC_TAG(1 + h, 2, j));
        if (!all_visible) {
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int left = vis - 32 * q4;
            const uint32_t bits = left >= 32 ? 0xffffffffu : (left <= 0 ? 0u : ((1u << left) - 1u));
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!((bits >> i) & 1u)) sv[32 * q4 + i] = 0xff800000u;   // -inf
          }
        }
        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < BN; i += 8) {
          mx4[0] = max3_nan(mx4[0], __uint_as_float(sv[i]), __uint_as_float(sv[i + 1]));
          mx4[1] = max3_nan(mx4[1], __uint_as_float(sv[i + 2]), __uint_as_float(sv[i + 3]));
          mx4[2] = max3_nan(mx4[2], __uint_as_float(sv[i + 4]), __uint_as_float(sv[i + 5]));
          mx4[3] = max3_nan(mx4[3], __uint_as_float(sv[i + 6]), __uint_as_float(sv[i + 7]));
        }
        const float mx = scaled_maximum(max3_nan(max_nan(mx4[0], mx4[1]), mx4[2], mx4[3]), p.scale_log2e);   // scale > 0
        const float m_new = max_nan(m_used, mx);

        // P = 2^(s * scale - ref) as bf16 pairs over the scores (masked: 2^-inf = 0), 64 keys at a time.  The row sum takes P before its
        // rounding.  The exponential unit takes 8 cycles per warp and instruction, as long for a tile as the tensor pipe, so a
        // share of the keys takes the polynomial -- where all keys are visible and no row's reference is infinite, NaN or coarse.
        uint64_t sum2[2] = {0ull, 0ull};
        auto weights = [&](auto half_tag, auto poly_tag, float scale, float neg_ref) {
          constexpr int kHalf = decltype(half_tag)::value, kPoly = decltype(poly_tag)::value;
          const uint64_t scale2 = pack_f32x2(scale, scale), ref2 = pack_f32x2(neg_ref, neg_ref);
#pragma unroll
          for (int c = kHalf ? kFirstChunks : 0; c < (kHalf ? 4 : kFirstChunks); ++c) {
            uint32_t pk[16];
            uint64_t xs[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
              xs[i] = fma_f32x2(pack_f32x2(__uint_as_float(sv[32 * c + 2 * i]), __uint_as_float(sv[32 * c + 2 * i + 1])), scale2, ref2);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if ((i + 1) * kPoly / 16 > i * kPoly / 16) {
                xs[i] = exp2_poly2(xs[i]);
              } else {
                float p0, p1;
                unpack_f32x2(xs[i], p0, p1);
                xs[i] = pack_f32x2(fast_exp2(p0), fast_exp2(p1));
              }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float p0, p1;
              sum2[i & 1] = add_f32x2(sum2[i & 1], xs[i]);
              unpack_f32x2(xs[i], p0, p1);
              pk[i] = pack_bf16x2(p0, p1);
            }
            tmem_st16(t_s + uint32_t(c) * 16u, pk);
          }
        };
        auto publish = [&](int half) {
          tmem_wait_st();
          tc_fence_before();
          named_arrive(kBarP + 2 * h + half, kPCount);
          trace_event(trace, DYSPEC_TAG(1 + h, 4 + half, j));
        };
        constexpr std::integral_constant<int, 0> kFirst{}, kExact{};
        constexpr std::integral_constant<int, 1> kSecond{};
        constexpr std::integral_constant<int, kPolyPairs<D>> kMixed{};
        // The reference almost always stays: the first weights are computed against the one there is, beside the maximum
        // instead of behind it, and again in the rare tile that raises it.
        // (Rows that are not the request's have no vote: what their Q holds changes no bit of the others.)
        const bool raised = ok && !(m_new <= m_used + kRescaleThreshold);
        bool careful = j == 0 || !all_visible || !__all_sync(0xffffffffu, !ok || fabsf(m_used) <= kCoarseReference);
        if (!careful) {
          weights(kFirst, kMixed, p.scale_log2e, -m_used);
          careful = __any_sync(0xffffffffu, raised);
        }
        trace_event(trace, DYSPEC_TAG(1 + h, 3, j));
        if (!careful) {
          publish(0);
          weights(kSecond, kMixed, p.scale_log2e, -m_used);
        } else {
          if (j == 0) {
            m_used = m_new;
          } else if (__any_sync(0xffffffffu, raised)) {
            // rescale the running output of this warp's 32 rows: O *= 2^(m_used - m_new)  (P V(j - 1) is done, see above)
            const float f = fast_exp2(m_used - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t v[32];
              tmem_ld32(t_o + uint32_t(c) * 32u, v);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
              tmem_st32(t_o + uint32_t(c) * 32u, v);
            }
            l *= f;
            m_used = m_new;
          }
          // V rows behind the end of the sequence are not ours: zero them (their probabilities are 0, but 0 * garbage could be
          // NaN), a row per thread, chunks in an order that spreads the banks.  Both halves do, each before it publishes its P:
          // neither's product waits for the other half.
          if (own < BN) {
            const uint32_t at = ring0 + 2u * uint32_t(j) + 1u, vslot = at % kSlots;
            mbar_wait_idle(bar(Br::kSlotFull + vslot), (at / kSlots) & 1u, abort_flag, p.status);
            if (r >= own) {
              uint8_t* v_row = smem + L::kRingOffset + vslot * L::kTileBytes + r * 128;
#pragma unroll
              for (int i = 0; i < 8 * L::kPanels; ++i)
                *reinterpret_cast<uint4*>(v_row + (i >> 3) * L::kPanelBytes + ((r + i) & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
            __syncwarp();
          }
          sum2[0] = sum2[1] = 0ull;
          const float scale = scale_for_reference(m_used, p.scale_log2e);
          const float neg_ref = m_used == -INFINITY ? 0.f : -m_used;
          weights(kFirst, kExact, scale, neg_ref);
          publish(0);
          weights(kSecond, kExact, scale, neg_ref);
        }
        publish(1);
        float a0, a1, b0, b1;
        unpack_f32x2(sum2[0], a0, a1);
        unpack_f32x2(sum2[1], b0, b1);
        l += (a0 + a1) + (b0 + b1);
      }

      // ---- epilogue: wait for the last P V, read O, normalise (or emit the partial)
      mbar_wait_idle(bar(Br::kODone + h), n_o & 1u, abort_flag, p.status);
      ++n_o;
      __syncwarp();
      tc_fence_after();
      trace_event(trace, DYSPEC_TAG(1 + h, 6, 0));
      if (!dep_ok) {
        grid_dependency_wait();                            // global writes from here on
        dep_ok = true;
      }
      if (item.slot < 0) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        __nv_bfloat16* out = p.out + (size_t(item.node0 + token) * p.n_q_heads + item.kv_head * g + (row & (g - 1))) * D;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(t_o + uint32_t(c) * 32u, v);
          tmem_wait_ld();
          if (c == D / 32 - 1) { tc_fence_before(); mbar_arrive(bar(Br::kOFree + h)); }
          if (ok) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) pk[i] = pack_bf16x2(__uint_as_float(v[2 * i]) * inv, __uint_as_float(v[2 * i + 1]) * inv);
            st_global_row16(out + c * 32, pk, wide_rows(p.out));
          }
        }
      } else {
        // partial slot: O [256][D] fp32, then m [256], then l [256]
        float* slot_at = p.partial + size_t(item.slot) * p.slot_floats;
        const int pr = h * BMH + r;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(t_o + uint32_t(c) * 32u, v);
          tmem_wait_ld();
          if (c == D / 32 - 1) { tc_fence_before(); mbar_arrive(bar(Br::kOFree + h)); }
          if (ok) {
#pragma unroll
            for (int i = 0; i < 4; ++i) st_global_v8(slot_at + pr * D + c * 32 + 8 * i, v + 8 * i);
          }
        }
        if (ok) {
          slot_at[2 * BMH * D + pr] = m_used;
          slot_at[2 * BMH * D + 2 * BMH + pr] = l;
        }
      }
      trace_event(trace, DYSPEC_TAG(1 + h, 7, 0));
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

namespace {
template <int D>
cudaError_t launch_one(cudaLaunchConfig_t& cfg, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv,
                       const AttnParams& p, const FirstItems& first) {
  static DynSmemGrant grant;           // one per instantiation
  // (padded past half of an SM's shared memory: one CTA per SM, since each CTA takes all 512 TMEM columns)
  const size_t smem = CausalLayout<D>::kTotal + 1024 > 120 * 1024 ? CausalLayout<D>::kTotal + 1024 : 120 * 1024;
  if (cudaError_t e = grant.ensure(causal_attn_kernel<D>, smem); e != cudaSuccess) return e;
  cfg.dynamicSmemBytes = smem;
  return cudaLaunchKernelEx(&cfg, causal_attn_kernel<D>, mq, mk, mv, p, first);
}
}  // namespace

cudaError_t launch_attn_causal(int head_dim, int n_ctas, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv,
                               const AttnParams& p, const WorkItem* host_items, cudaStream_t stream) {
  FirstItems first;                    // host_items: the host copy of p.items; each CTA's first item travels as a kernel parameter
  for (int c = 0; c < kFirstItems; ++c) first.item[c] = c < n_ctas ? host_items[c] : WorkItem{};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(n_ctas));
  cfg.blockDim = dim3(unsigned(kThreads));
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = head_dim == 128 ? launch_one<128>(cfg, mq, mk, mv, p, first) : launch_one<64>(cfg, mq, mk, mv, p, first);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace dyspec
