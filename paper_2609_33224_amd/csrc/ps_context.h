// The context behind the C ABI, and what its entry points share.
#pragma once

#include <string>
#include <vector>

#include "ps_device.h"

using namespace ps;  // (the context is a C type)

struct ps_ctx {
  int device = 0;
  hipStream_t stream = nullptr;
  // the scoring call's second stream (the walk pass, beside the popular
  // pass on the calling stream) and the events of its fork and join
  hipStream_t aux = nullptr;
  hipEvent_t fork_ev = nullptr, join_ev = nullptr;
  int num_cus = 0;
  std::string err;
  DevPool pool;  // all device memory of the context
  bool loaded = false;
  // snapshot
  int32_t n_inst = 0;
  int32_t cap = 0;
  Tables t{};
  InstState* d_inst = nullptr;
  int64_t* d_room = nullptr;
  int64_t* d_room_sorted = nullptr;
  uint32_t* d_order0 = nullptr;
  InstState* d_inst_key = nullptr;  // states in d_order0's order
  TopRoom* d_rtop = nullptr;         // the kTopRooms largest rooms with their ids
  uint32_t* d_rank = nullptr;        // ranks of the derivation (2 per instance)
  int32_t lean_wpc = 0;              // resident lean-scorer waves per CU (0: not asked yet)
  int32_t rows_wpc = 0;              // the same for the four-requests-per-wave scorer
  int32_t score_wpc = 0;             // the same for the general scorer (fast policy)
  int4* d_lm = nullptr;              // zero-hit admission thresholds in that order
  int32_t* d_lm1 = nullptr;          // their maxima per 64 positions
  uint4* d_csum = nullptr;           // per 64 positions: least t_iter (A1 > 1, A1 <= 1), largest room
  GIndex x{nullptr, nullptr, nullptr, 0, 0, 64};
  DevModel* d_model = nullptr;
  unsigned long long* d_counter = nullptr;  // a call's count, then its first zero hash
  uint16_t* d_scratch = nullptr;
  int scratch_rows = 0;
  bool hits_in_lds = true;
  std::vector<InstState> h_state;
  std::vector<uint32_t> h_count;
  DevModel h_model{};
  // feedback: EMA factors in double between updates; recent output lengths
  std::vector<double> gamma64;
  std::vector<int32_t> lout_ring;
  int64_t lout_seen = 0;
  float lout_raw = 0.0f;
  // staging for the host-memory entry points
  void* d_stage[3] = {nullptr, nullptr, nullptr};
  size_t stage_cap[3] = {0, 0, 0};
  // per-arrival scheduler: hits of one launch's requests on every instance
  uint32_t* d_seq_hits = nullptr;
  size_t seq_hits_cap = 0;  // bytes
  SpecRec* d_spec = nullptr;  // a launch's speculative results
  int32_t spec_cap = 0;       // records
  size_t seq_budget = (size_t)256 << 20;  // bytes of hits per scheduler launch
  // speculative batches (requests per batch; 0: every request scored in full)
  int32_t spec_batch = kSpecBatch;
  // chain positions of a commit's slice and of a scheduling batch at most
  int64_t max_pos = kCommitMaxPos;
  unsigned long long* d_seq_stats = nullptr;     // decisions from speculation, scored in full
  // prefix groups of the scored windows: slot keys (tagged with a window
  // generation, so a new window needs no clearing), slot records, and each
  // request's slot
  unsigned long long* d_gkeys = nullptr;  // keys, then the tagged segment lengths
  uint2* d_grec = nullptr;
  uint32_t* d_gslot = nullptr;
  uint32_t* d_gpop = nullptr;  // kGroupHeadWords counter words (rows taken, deferral; two sets
                               // of leader list lengths, one 128-byte line per list), then
                               // the popular rows
  unsigned long long* d_glist = nullptr;  // the leaders' lists (kXcds * glcap)
  uint32_t glcap = 0;           // entries per list
  uint32_t gslots = 0;   // power of two
  int32_t greq_cap = 0;  // entries of d_gslot
  // the rows scorer's hand-over: kDeferLists sub-list lengths (one 128-byte
  // line each) and the sub-lists (dcap entries each)
  uint32_t* d_dcnt = nullptr;
  int32_t* d_dlist = nullptr;
  int64_t dcap = 0;
  uint64_t ggen = 0;
  bool gclear = false, grep_clear = false;  // to be cleared before the next window's launches
  uint2* d_gplist = nullptr;  // the popular pass's groups
  uint32_t gplist_cap = 0;
  unsigned long long* d_grep = nullptr;  // representatives, per holder bitmap
  uint32_t grep_cap = 0;
  uint32_t* d_gpre = nullptr;            // prefix rows (grep_cap x n_inst), then grep_cap ends
  size_t gpre_cap = 0;                   // words
  // order of the exhaustive probe's requests (counting-sort bins, order)
  uint32_t* d_obins = nullptr;
  int32_t* d_order = nullptr;
  int32_t order_cap = 0;
  // optional per-launch timing of the scoring path: events recorded on the
  // call's stream before the group pass, between it and the scoring kernel,
  // and after it, for up to kTimingCalls calls
  bool timing = false;
  int32_t n_timed = 0;
  std::vector<hipEvent_t> ev;  // 3 per call
  ps_attend_plan* plans = nullptr;  // the attention plans of the context, a list
};

namespace ps {

// Sets the message of ps_last_error and returns `code`.
ps_status fail(ps_ctx* c, ps_status code, const char* fmt, ...) __attribute__((format(printf, 3, 4)));

// Frees the context's attention plans (ps_destroy).
void free_plans(ps_ctx* c);

#define HIP_TRY(ctx, call)                                                                  \
  do {                                                                                      \
    hipError_t e_ = (call);                                                                 \
    if (e_ != hipSuccess)                                                                   \
      return fail(ctx, e_ == hipErrorOutOfMemory ? PS_E_NOMEM : PS_E_DEVICE, "%s: %s", #call, \
                  hipGetErrorString(e_));                                                   \
  } while (0)

// Makes ctx's device current for the scope of an entry point.
struct DeviceScope {
  int prev = -1;
  explicit DeviceScope(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    if (prev != dev) (void)hipSetDevice(dev);
  }
  ~DeviceScope() {
    int cur = -1;
    if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

}  // namespace ps
