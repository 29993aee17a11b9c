"""How the attentions over a 4-bit cache end when a wait has run out somewhere: nothing is read that nobody wrote, no lane is left
behind, no copy is left in flight.  The functions run on the host (see _warp_emulation); no GPU, and no fault anywhere."""
import re

import pytest

from tests import _warp_emulation as emu

# Stand-ins for what the decoders call: copies that are never waited for, a cache of one block, loads that know what they may read.
DECODERS = r'''
constexpr int kTile = 128, kWarps = 12, kDecoders = 4, kTallDecoders = 8, kUnitRing = 4, kNarrowRows = 16;
constexpr uint32_t kScaleLeast = 0, kScaleMost = 0;
struct Q4Cache { uint8_t* data; int64_t s_page, s_head; };
thread_local uint8_t* my_smem;
alignas(16) uint8_t published[17 * 128];
int bad_loads = 0;
template <typename T>
inline T __ldcg(const T* p) {
  const uint8_t* at = reinterpret_cast<const uint8_t*>(p);
  if (at < published || at + sizeof(T) > published + sizeof(published)) { ++bad_loads; return T{}; }
  return *p;
}
inline uint32_t smem_u32(const void*) { return 0; }
inline void fence_async_smem() {}
int arrivals = 0;
inline void mbar_arrive(uint32_t) { ++arrivals; }
inline bool mbar_wait(uint32_t, uint32_t, const Abort&, int, long long = 0) { return true; }     // the slot is free
'''


def decoders():
    src = emu.text("tree_attn.cu")
    parts = [DECODERS, emu.definition(emu.text("q4.cuh"), r"^template <int D>\nstruct Block \{"), emu.definition(src, r"^template <int D>\nstruct Plan \{"),
             emu.definition(src, r"^template <int BLOCKS>\nstruct Coded \{"), "template <int D> inline void decode_run(const uint4&, uint32_t, uint32_t, int, int) {}\n"]
    if "bool warp_wait(" in src:
        parts.append(emu.definition(src, r"^template <typename There>\n__device__ __forceinline__ bool warp_wait\("))
    parts.append(emu.definition(src, r"^template <int D>\n__device__ __forceinline__ const uint8_t\* volatile\* block_ring\("))
    parts.append(emu.definition(src, r"^template <int D, int BLOCKS>\n__device__ __noinline__ void decode\("))
    return "\n".join(parts) + r'''
// Shared memory of a CTA whose first `found` tiles have been looked up; the other tiles' addresses are what lay there.
struct Memory {
  std::vector<uint8_t> bytes = std::vector<uint8_t>(Plan<DIM>::TOTAL, 0xee);
  int flag = 0, status[2] = {0, 0};
  explicit Memory(int found) { *ready() = found; for (int i = 0; i < 8; ++i) ready()[1 + i] = 0; for (int t = 0; t < found; ++t) publish(t); }
  int* ready() { return reinterpret_cast<int*>(bytes.data() + Plan<DIM>::PROGRESS_OFF); }
  void publish(int t) { for (int b = 0; b < 8; ++b) block_ring<DIM>(bytes.data(), t)[b] = published; }
};
'''


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("blocks,lead", [(1, 2), (2, 1)], ids=["tall", "wide"])
@pytest.mark.parametrize("found", [1, 2, 3, 4, 5, 6, 7])
def test_a_decoder_that_stops_reads_no_address_that_nobody_wrote(tmp_path, dim, blocks, lead, found):
    """Another CTA's timeout stops the look-up after `found` tiles while every slot of the ring is free."""
    emu.run(tmp_path, f"constexpr int DIM = {dim};\n" + decoders() + f'''
int main() {{
  Memory m({found});
  m.flag = 1;
  run_lanes(2, [&](int lane) {{
    threadIdx.x = kWarps * 32 + lane;
    Q4Cache cache{{published, 0, 0}};
    decode<{dim}, {blocks}>(cache, m.bytes.data(), 0, Abort{{&m.flag, m.status}}, 100, {lead});
  }});
  if (bad_loads) fail("loads through addresses that were never looked up");
  if (m.ready()[1] > {found}) fail("more tiles counted as fetched than were looked up");
  std::puts("ok");
}}
''')


@pytest.mark.parametrize("found", [1, 2, 3, 4, 7])
def test_lanes_of_a_decoder_stop_together(tmp_path, found):
    """One lane still sees the last look-up, another one already the flag."""
    emu.run(tmp_path, "constexpr int DIM = 128;\n" + decoders() + f'''
int main() {{
  Memory stops({found}), goes({found} + 1);
  stops.flag = 1;
  run_lanes(2, [&](int lane) {{
    threadIdx.x = kWarps * 32 + lane;
    Memory& m = lane == 0 ? goes : stops;
    if (lane == 0) goes.flag = 1;
    Q4Cache cache{{published, 0, 0}};
    decode<128, 1>(cache, m.bytes.data(), 0, Abort{{&m.flag, m.status}}, 100, 2);
  }});
  if (bad_loads) fail("loads through addresses that were never looked up");
  std::puts("ok");
}}
''')


def test_a_decoder_does_not_wait_for_ever(tmp_path):
    """Nobody looks anything up and nobody raises the flag: the decoder does, after its limit, with a timeout in the status word."""
    emu.run(tmp_path, "constexpr int DIM = 128;\n" + decoders() + '''
int main() {
  Memory m(2);
  run_lanes(2, [&](int lane) {
    threadIdx.x = kWarps * 32 + lane;
    Q4Cache cache{published, 0, 0};
    decode<128, 1>(cache, m.bytes.data(), 0, Abort{&m.flag, m.status}, 100, 2);
  });
  if (bad_loads || !m.flag || m.status[0] != SP_ERR_TIMEOUT) fail("no timeout");
  std::puts("ok");
}
''', 100)


def test_a_decoder_that_nothing_stops_takes_every_tile(tmp_path):
    emu.run(tmp_path, "constexpr int DIM = 128;\n" + decoders() + '''
int main() {
  Memory m(8);
  *m.ready() = 20;
  run_lanes(2, [&](int lane) {
    threadIdx.x = kWarps * 32 + lane;
    Q4Cache cache{published, 0, 0};
    decode<128, 1>(cache, m.bytes.data(), 0, Abort{&m.flag, m.status}, 20, 2);
  });
  if (bad_loads || m.flag || m.ready()[1] != 20 || arrivals != 40) fail("tiles left out");
  std::puts("ok");
}
''')


# Stand-ins for what a producer lane calls: a run of one piece, copies that land some polls of their barrier after they were issued.
PRODUCER = r"""
struct TreeAttnArgs { const int32_t* table; int max_pages, page_log2, n_pages; int* status; };
struct Q4Cache { uint8_t* data; int64_t s_page, s_head; };
constexpr int kWhereTreePageQ4 = 71;
struct Plan1 { static constexpr int ROWS = 8, KEYS = 32, BLOCK = 17 * 128, BYTES = 2 * BLOCK, RING = 3, RING_OFF = 0, BAR_OFF = 1 << 20; };
template <int D, int NT> using Plan = Plan1;
struct Request { int start, n, len, past, kt; };
struct Piece { int start, r0, rows, g, b, len, past, kt0, n, kt_all; };
struct Walk { long long rem, left; int b; Request q; };
int steps = 0, issued[3], landed[3], released[3], polls = 0, slow = 0, gives_up_at = 1 << 30;
volatile int abort_flag = 0;
template <int ROWS, int KEYS>
bool walk_on(const TreeAttnArgs&, Walk& w, Piece& u) {
  if (w.left <= 0) return false;
  u.b = u.g = 0; u.len = (int)w.left * 32; u.kt0 = 0; u.n = (int)w.left;
  w.left = 0;
  return true;
}
inline void mbar_expect_tx(uint32_t bar, uint32_t) { ++issued[(bar - Plan1::BAR_OFF) / 16 % 3]; }
inline void bulk_copy(uint32_t, const void*, uint32_t, uint32_t) {}
inline bool mbar_test(uint32_t bar, uint32_t parity) {
  const int slot = (bar - Plan1::BAR_OFF) / 16 % 3;
  ++polls;
  if (bar & 8) {                   // free: the consumer has read what landed, until it gives up
    if (issued[0] + issued[1] + issued[2] >= gives_up_at) { abort_flag = 1; return false; }
    landed[slot] = issued[slot];
    return true;
  }
  if (slow >= 0 && polls > slow && landed[slot] < issued[slot]) { polls = 0; ++landed[slot]; }
  return (uint32_t)(landed[slot] & 1) != parity;
}
inline bool mbar_try_wait(uint32_t bar, uint32_t parity) { return mbar_test(bar, parity); }
"""


@pytest.mark.parametrize("steps,gives_up,slow", [(1, 99, 9), (2, 99, 9), (3, 99, 9), (20, 99, 9), (20, 7, 9), (20, 3, 9), (0, 99, 9), (3, 99, -1), (20, 7, -1)])
def test_a_producer_leaves_no_copy_in_flight(tmp_path, steps, gives_up, slow):
    """Whether it has issued all of its copies or met the abort flag: they have landed when it returns, as a warp that gives up after
    that ends the CTA at once.  (slow -1: they never land; it returns all the same.)"""
    emu.run(tmp_path, PRODUCER + emu.definition(emu.text("q4_attn.cu"), r"^template <int D, int NT>\n__device__ __noinline__ void produce\(") + f"""
int main() {{
  int status[2] = {{0, 0}}, table[64] = {{}};
  uint8_t data[16];
  slow = {slow}; gives_up_at = {gives_up}; tick = 1000;
  run_lanes(1, [&](int) {{
    produce<128, 1>(TreeAttnArgs{{table, 64, 5, 1, status}}, Q4Cache{{data, 0, 0}}, 0, Abort{{&abort_flag, status}}, Walk{{0, {steps}, 0, Request{{}}}}, 0);
  }});
  for (int i = 0; i < 3; ++i)
    if (slow >= 0 && landed[i] != issued[i]) fail("a copy is still in flight");
  if (issued[0] + issued[1] + issued[2] != std::min({steps}, {gives_up})) fail("not all copies were issued");
  std::puts("ok");
}}
""")


@pytest.mark.parametrize("name", ["q4_attn.cu", "tree_attn.cu"])
def test_the_status_word_is_voted_on_before_anything_depends_on_it(name):
    """Each thread reads the status word for itself, and another kernel may write it in between: what threads with barriers and votes
    ahead of them do about it is the same for the whole CTA.  (A thread that ends at once, as in the other kernels, is waited for nowhere.)"""
    src = re.sub(r"//.*", "", emu.text(name))
    own = re.findall(r"\b(\w+) = decode_poisoned\(", src)
    ends = re.findall(r"if \(decode_poisoned\([^)]*\)[^;]*\) return;", src)
    assert own and len(own) + len(ends) == src.count("decode_poisoned(")
    for var in own:
        uses = re.findall(rf"[^\n]*\b{var}\b[^\n]*", src)
        assert len(uses) == 2 and "__syncthreads_or(" in uses[1], uses


@pytest.mark.parametrize("name", ["tree_attn.cu", "attn_tc.cu"])
def test_other_producers_wait_for_their_copies_whether_or_not_the_flag_is_up_yet(name):
    """(The paired kernel's producer waits for each copy as it relays it, so that only a run that it broke off itself leaves any.)"""
    src = emu.text(name)
    at = [m.start() for m in re.finditer("let the copies already in flight land", src)]
    assert at
    for x in at:
        condition = [line for line in src[:x].splitlines()[:-1] if line.strip()][-1]
        assert "abort_flag" not in condition, condition
