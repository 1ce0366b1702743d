// Host-side planning of one hybrid-batch iteration (no HIP calls).
//
// Turns a batch descriptor into the int32 metadata the kernels read: per-token
// position and request, per-request block-table offset, the block ids, the
// attention work list and the split-merge groups. Everything is packed into
// one array so one host-to-device copy moves it.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

#include "hb.h"

namespace hb {

// Set the thread-local message returned by hb_last_error(); returns `st`.
hb_status fail(hb_status st, const char* fmt, ...);
const char* last_error();
// The status of a C entry that caught std::bad_alloc: no exception leaves one.
hb_status host_oom();

struct Dims {
  int H = 0, nq = 0, nkv = 0, hd = 0, F = 0, blk = 16;
  int G = 0;      // q heads per kv head
  int P = 0;      // query positions of a 16-column wave item = 16 / G
  int BQ = 0;     // query positions of a workgroup tile = kTileCols / G
  int qkv_n = 0;  // (nq + 2 nkv) * hd
  float theta = 0.f, eps = 0.f;
  int max_T = 0, max_R = 0;
};

// Bytes of an operand the GEMMs can address: each operand is read through a
// raw buffer resource of this many records (and 32-bit byte offsets), so
// nothing past it may be needed. Rows past M that the GEMMs read from their
// activation operands (whole row tiles): kGemmPadRows.
constexpr int64_t kOperandWindow = 0x7FFFFFF0;
constexpr int kGemmPadRows = 512;

hb_status check_config(const hb_layer_config* cfg, Dims* d);

// HB_ERR_UNSUPPORTED unless rows x cols bf16 values fit the operand window.
hb_status check_window(const char* what, int64_t rows, int64_t cols);

// Rows of `width` elements, `stride` apart.
struct Rows {
  uintptr_t at;
  int64_t stride, width;
  uintptr_t end(int T) const { return at + ((uintptr_t)(T - 1) * stride + width) * 2; }
};
// The arguments of hb_run_append (T > 0 rows), hb_set_attention_rope and hb_sample.
hb_status check_append(const Dims& d, int num_blocks, int T, const hb_kv_pool* pool, const Rows& q, const Rows& k,
                       const Rows& v, const Rows& out);
hb_status check_rope(int head_dim, int rotary_dim, int layout, const double* inv_freq, double magnitude);
hb_status check_sample(int max_rows, int vocab, const hb_sample_desc* desc);

// Sliding window with sinks. A row at position p sees key j <= p when
// j > p - window or j < sinks (window 0: every j <= p).
struct Window {
  int window = 0, sinks = 0;
  bool operator==(const Window& o) const { return window == o.window && (window == 0 || sinks == o.sinks); }
};
hb_status check_window_args(int window, int sinks);

// Blocks [first, first + count) of a table that no row at a position >= pos
// sees: past the sinks' last block, before the block of key pos - window + 1.
struct DeadBlocks {
  int first = 0, count = 0;
};
DeadBlocks dead_blocks(const Window& w, int pos);

// Attention work over the key positions [kv_begin, kv_end) of one request
// and kv head: a wave item covers 16 query columns (P positions x G heads), a
// workgroup tile kTileCols columns (BQ positions x G heads). part < 0: the unit
// writes the normalised output; otherwise its columns' partial results go to
// column slots part + c.
struct AttnItem {
  int32_t req, kv_head, tok0, pos0, npos, kv_begin, kv_end, part;
};
// Where a windowed unit's axis block i stands in its request's uploaded table:
// i + sink below Plan.sink_blocks, i + window from there on (the upload leaves
// out the blocks that no row of the request sees, and req_bt points as if it
// had not).
struct UnitShift {
  int32_t sink, window;
};
// Columns whose key range was split: part s of column c sits in slot
// part0 + s * stride + c.
struct MergeGroup {
  int32_t part0, nparts, stride, tok0, npos, kv_head;
  int32_t cols;  // a merge record's: its block of 16 of the columns
  int32_t pad;
};
static_assert(sizeof(AttnItem) == 32 && sizeof(MergeGroup) == 32, "packed as 8 int32");
static_assert(sizeof(UnitShift) == 8, "packed as 2 int32");

// Each request's block ids are followed by kBtPad copies of its last id, so
// the four ids of a 64-key step can be read as one vector even at the end.
constexpr int kBtPad = 3;
// Query columns of a workgroup tile (32 per wave), and wave items grouped to
// a workgroup (one per wave): the attention workgroup has 4 waves.
constexpr int kTileCols = 128;
constexpr int kItemsPerUnit = 4;
// One wave's work in one record, as hb_attention uploads it: four per
// workgroup, in launch order, so that a wave has all it needs for its first
// loads after one scalar load (units -> items -> req_bt -> bt otherwise).
enum { kRecTile = 0, kRecSingle = 1, kRecMerged = 2 };
struct UnitRec {
  AttnItem item;  // of the tile, or the wave's own
  int32_t kind;
  // axis block i stands at bt[sink + i] below Plan.sink_blocks (windowed plans)
  // and at bt[window + i] from there on
  int32_t sink, window, pad;
  // a tile's wave w: the blocks it copies in steps 0 .. 3 (block w % 2 of each);
  // an item's: both blocks of steps 0 and 1 (past the range: its last block)
  int32_t ids[4];
};
static_assert(sizeof(UnitRec) == 64, "packed as 16 int32");

// Work unit encoding: u >= 0 is tile u; -1 - v runs items 4 w .. 4 w + 3 with
// w = v & ~kUnitMerged, one per wave. Without kUnitMerged the four items are
// independent. With it they are consecutive key ranges of one (request, kv
// head, query positions), possibly empty (kv_begin == kv_end): the workgroup
// combines them in LDS and writes one result, to the output when item 4 w's
// part is < 0, else to that part's column slots.
constexpr int32_t kUnitMerged = 1 << 29;

struct Plan {
  int T = 0, R = 0;
  int n_tiles = 0, n_items = 0, n_units = 0, n_groups = 0, n_merge_units = 0;
  int n_slots = 0;  // partial-result column slots
  bool too_many_slots = false;  // a shared plan of more than 2^30 of them, which cannot run
  int split_tile = 0, split_item = 0;
  // some row's window hides a key from it: the units have shifts, and the
  // kernels that apply `window` run
  bool windowed = false;
  bool paired = false;  // item units alone, but for one round of two workgroups per CU
  bool half_tiles = false;  // tiles of kTileCols / 2 columns (a plan of records)
  Window window;
  int sink_blocks = 0;
  // offsets (int32 units) of each section inside meta
  int off_tok_pos = 0, off_tok_req = 0, off_req_bt = 0, off_bt = 0;
  int off_tiles = 0, off_items = 0, off_units = 0, off_groups = 0, off_merge = 0;
  int off_tile_shift = 0, off_item_shift = 0;
  std::vector<int32_t> meta;
  // algorithmic work of the iteration (for roofline accounting)
  double flops = 0, bytes = 0;
};

// Scratch reused across calls for the duplicate-slot check.
struct SlotMarks {
  std::vector<uint16_t> mask;    // per block: bit o set when slot o is written
  std::vector<int32_t> touched;  // blocks to clear afterwards
};

// Validate `desc` against the layer shape and a pool of num_blocks blocks. Table
// entries that the window hides from every row of their request are not looked at.
hb_status check_batch(const Dims& d, int num_blocks, const hb_batch_desc* desc, SlotMarks* marks,
                      const Window& w = Window());
// The part of it that concerns the requests alone; *n_tokens receives their rows.
// skip: leading table entries of each request that are not looked at, or null.
hb_status check_requests(const Dims& d, int num_blocks, const hb_request* requests, int n, const Window& w,
                         int64_t* n_tokens, const std::vector<int>* skip = nullptr);
// The part of it that forbids two requests to write one slot (of checked requests).
hb_status check_slots(int num_blocks, const hb_request* requests, int n, int64_t n_tokens, SlotMarks* marks);
// Requests (checked by this, too) and the groups of them that share a prefix.
hb_status check_shared(const Dims& d, int num_blocks, const hb_request* requests, int n, const hb_prefix_group* groups,
                       int n_groups, int64_t* n_tokens);

// Fixed split lengths (keys, multiples of 64; 0 = chosen from the batch),
// for tuning and tests.
struct PlanOptions {
  int split_tile = 0, split_item = 0;
  int min_item = 64;   // least item split the planner chooses by itself
  int unit_block = 0;  // runs of tiles / item groups in the unit order (0: one per CU; < 0: fine interleave)
  Window window;
  // As hb_attention plans (layers do not). Launches that need one round of
  // workgroups at most are cut for that round: item ranges are split for it, small
  // launches with chunks take no tiles (their units in the order by die), few tiles
  // are halved or split. And where items are few, in launches of any size, no wave
  // takes more than 256 keys alone.
  bool fit_round = false;
  // groups of requests that share a prefix (checked; no window then)
  const hb_prefix_group* groups = nullptr;
  int n_groups = 0;
  bool share_all = false;  // join however short a prefix is (testing)
};

// Build the plan of a validated batch for a GPU with cu_count compute units.
void build_plan(const Dims& d, const hb_batch_desc* desc, int cu_count, Plan* p,
                const PlanOptions& opt = PlanOptions());

// A plan as hb_attention uploads it: 4 n_units records, then the plan's block
// ids and a merge record (the group, with its block of columns) per merge unit,
// at these offsets (int32).
struct RecordPlan {
  int off_bt = 0, off_merge = 0;
  std::vector<int32_t> meta;
};
void build_records(const Plan& p, RecordPlan* out);

// New tokens of one request that go to one pool block: rows tok0 .. tok0 + n - 1
// at positions pos0 .., slots pos0 % 16 .. of `block`.
struct AppendUnit {
  int32_t tok0, pos0, n, block;
};
static_assert(sizeof(AppendUnit) == 16, "packed as 4 int32");
// The batch's append units, behind what `out` holds; returns their number and their offset (int32).
int build_append(const hb_request* requests, int n, std::vector<int32_t>* out, int* off);

// Algorithmic flops and HBM bytes of one iteration (what the method must
// compute and move, not what an implementation happens to do).
void iteration_work(const Dims& d, const hb_request* reqs, int n, double* flops, double* bytes,
                    const Window& w = Window());

}  // namespace hb
