// Host side of the linear-attention entry points without a GPU (test code): their source is compiled for the host alone, under
// UndefinedBehaviorSanitizer, against a stand-in for the runtime that keeps the launches in place of running them.
#include "../paper_2002_03629_amd/csrc/linattn.hip"

#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>

struct Launch {
  std::string kernel;
  dim3 grid, block;
  LinattnArgs args;
};
static std::vector<std::pair<const void*, std::string>> g_names;
static std::vector<Launch> g_launches;
static dim3 g_grid, g_block;
static char g_error[512];

int jm::fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_error, sizeof g_error, fmt, ap);
  va_end(ap);
  return code;
}

extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* fn, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  g_names.emplace_back(fn, name);
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid;
  g_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = g_grid;
  *block = g_block;
  *shared = 0;
  *stream = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* fn, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  Launch l;
  for (auto& n : g_names)
    if (n.first == fn) l.kernel = n.second;
  l.grid = grid;
  l.block = block;
  memset(&l.args, 0, sizeof l.args);
  if (l.kernel.find("step") == std::string::npos) l.args = *(const LinattnArgs*)args[0];
  g_launches.push_back(l);
  return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return ""; }
}

static int failures = 0;
#define EXPECT(cond, ...)                                                     \
  do {                                                                        \
    if (!(cond)) { printf("line %d: %s: ", __LINE__, #cond); printf(__VA_ARGS__); printf("\n"); ++failures; } \
  } while (0)

static char g_memory[64 * 256];                        // places that no call follows
template <typename T>
static T* at(int i) { return (T*)((((uintptr_t)g_memory + 255) / 256 + i) * 256); }

static linattn_config config(int B, int T, int heads, int kv, int Dk, int Dv, int dtype, const int* offsets) {
  linattn_config c;
  memset(&c, 0, sizeof c);
  c.B = B;
  c.T = T;
  c.heads = heads;
  c.kv_heads = kv;
  c.Dk = Dk;
  c.Dv = Dv;
  c.dtype = dtype;
  c.scale = 1.0f;
  c.offsets = offsets;
  return c;
}

// One call with the workspace that it asks for (or none).
static int call(const linattn_config& c, bool backward, float* state_in, float* state_out, bool workspace = true) {
  int64_t bytes = 0;
  g_launches.clear();
  const int rc = linattn_workspace_bytes(&c, backward, &bytes);
  if (rc != MADE_OK) return rc;
  void* ws = workspace && bytes ? at<void>(0) : nullptr;
  if (!backward)
    return linattn_forward(&c, at<void>(1), at<void>(2), at<void>(3), at<float>(4), state_in, at<void>(5), state_out, ws, ws ? bytes : 0, nullptr);
  return linattn_backward(&c, at<void>(1), at<void>(2), at<void>(3), at<float>(4), state_in, at<void>(5), at<float>(6), at<void>(7), at<void>(8),
                          at<void>(9), state_out, ws, ws ? bytes : 0, nullptr);
}

// Where several workgroups read a sequence's state, none of them replaces it.
static void states_in_place() {
  int shared = 0;
  for (int dtype : {(int)MADE_F32, (int)MADE_BF16})
    for (bool packed : {false, true})
      for (int group : {1, 2, 3, 8})
        for (int kv : {1, 2, 8})
          for (int d : {16, 64, 128})
            for (bool workspace : {false, true}) {
              const std::vector<int> lengths = packed ? std::vector<int>{1, 0, 64, 700, 30, 1300, 5} : std::vector<int>{900, 900};
              std::vector<int> offsets = {0};
              for (int n : lengths) offsets.push_back(offsets.back() + n);
              const int B = (int)lengths.size(), T = packed ? offsets.back() : 900;
              const linattn_config c = config(B, T, group * kv, kv, d, d, dtype, packed ? offsets.data() : nullptr);
              float* state = at<float>(10);
              EXPECT(call(c, false, state, state, workspace) == MADE_OK, "%s", g_error);
              const LinattnArgs& a = g_launches.back().args;
              if (a.q_split > 1) ++shared;
              for (int b = 0; b < B; ++b) {
                LinattnPlace w;
                memset(&w, 0, sizeof w);
                w.s.count = std::max(1, (lengths[b] + a.seg_rows - 1) / a.seg_rows);
                w.state_at = (long long)b * kv * d * d;
                EXPECT(a.q_split == 1 || la_state_in(a, a.role[0], w) != a.role[0].end + w.state_at,
                       "dtype %d, packed %d, %d heads on %d states of %d, sequence of %d steps", dtype, packed, group * kv, kv, d, lengths[b]);
              }
            }
  EXPECT(shared > 20, "%d calls shared a state's heads", shared);
}

// Calls of many sequences, with the workspace that they ask for, are taken, and their launches are launches: within the limits of
// a grid, together over every state.  The states that the header promises: 8 million of width 128, 2.7 million for gradients.
static void many_sequences() {
  for (int backward : {0, 1})
    for (bool packed : {true, false})
      for (int dtype : {(int)MADE_F32, (int)MADE_BF16})
        for (int kv : {1, 32, 70000})
          for (int d : {16, 128})
            for (int B : {1, 300, 21845, 21846, 32767, 32768, 65535, 65536, 70000, 250000, 2700000, 8000000})
              for (int T : {0, 3, 200, 100000, 1 << 30}) {
                const long long states = (long long)B * kv;
                if (states > (backward ? 2700000 : 8000000) || (kv == 70000 && d == 128)) continue;
                static const int offsets[1] = {0};                  // (no call looks at it)
                const linattn_config c = config(B, T, kv, kv, d, d, dtype, packed ? offsets : nullptr);
                const int rc = call(c, backward, nullptr, at<float>(10));
                EXPECT(rc == MADE_OK, "%d sequences, %d steps, %d heads of %d, packed %d, dtype %d, backward %d: %s", B, T, kv, d, packed, dtype, backward, g_error);
                if (rc != MADE_OK) continue;
                const LinattnArgs& walk = g_launches.back().args;
                EXPECT(walk.roles == (backward ? 3 : 1) && (long long)walk.slots * kv * walk.q_split * walk.roles <= g_launches.back().grid.x, "%d sequences", B);
                long long joined = 0;
                bool join = false;
                for (const Launch& l : g_launches) {
                  EXPECT(l.grid.y <= 65535 && l.grid.z <= 65535 && l.grid.x > 0 && l.grid.y > 0 && l.grid.z > 0 &&
                             (double)l.grid.x * l.grid.y * l.grid.z * l.block.x < 4294967296.0,
                         "%s: %u x %u x %u workgroups", l.kernel.c_str(), l.grid.x, l.grid.y, l.grid.z);
                  if (l.kernel.find("join") == std::string::npos) continue;
                  join = true;
                  EXPECT(l.args.join0 == joined && (int)l.grid.x * 256 >= d * d && (int)l.grid.y == kv, "%lld joined", joined);
                  joined += l.grid.z;
                }
                EXPECT(joined == (join ? (long long)B * (backward ? 2 : 1) : 0) && (packed || !join || walk.seg_rows < T), "%lld joined", joined);
              }
}

// Every segment of a packed call has a number of its own, below the number of those that the call has room for.
static void segment_numbers() {
  unsigned seed = 1;
  auto draw = [&](int n) { return (int)((seed = seed * 1664525u + 1013904223u) >> 8) % n; };
  int cut = 0;
  for (int rep = 0; rep < 400; ++rep) {
    const int B = 1 + draw(rep % 4 ? 40 : 900), most = 1 << draw(12);
    std::vector<int> offsets = {draw(3)};
    for (int b = 0; b < B; ++b) offsets.push_back(offsets.back() + (draw(3) ? draw(most) : draw(2) * 64));
    const linattn_config c = config(B, offsets.back() + draw(2) * draw(200), 2, 2, 32, 32, rep % 2 ? MADE_BF16 : MADE_F32, offsets.data());
    EXPECT(call(c, rep / 2 % 2, nullptr, at<float>(10)) == MADE_OK, "%s", g_error);
    const LinattnArgs& a = g_launches.back().args;
    cut += a.role[0].seg != nullptr;
    int next = 0;
    for (int b = 0; b < B; ++b) {
      const int first = la_first_slot(a, b, offsets[b]);
      EXPECT(first >= next && (a.role[0].seg || first == b), "sequence %d of %d", b, B);
      next = first + la_count(a, offsets[b + 1] - offsets[b]);
    }
    EXPECT(next <= a.slots, "%d of %d", next, a.slots);
  }
  EXPECT(cut > 100, "%d calls were cut", cut);
}

int main() {
  states_in_place();
  segment_numbers();
  many_sequences();
  printf("%d failures\n", failures);
  return failures != 0;
}
