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
