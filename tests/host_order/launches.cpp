// Stand-ins for the HIP runtime's launch functions: loaded before libemb.so,
// they keep every kernel launch (name, grid, block) and run nothing.
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <map>
#include <string>
#include <vector>

struct Dim {
  uint32_t x, y, z;
};
struct Launch {
  std::string name;
  Dim grid, block;
};
static std::vector<Launch>& launches() {
  static std::vector<Launch> all;
  return all;
}
static std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> all;
  return all;
}
static Dim pushed_grid, pushed_block;
static size_t pushed_lds;
static void* pushed_stream;

extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
  names()[f] = name;
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t lds, void* stream) {
  pushed_grid = grid;
  pushed_block = block;
  pushed_lds = lds;
  pushed_stream = stream;
  return 0;
}
int __hipPopCallConfiguration(Dim* grid, Dim* block, size_t* lds, void** stream) {
  *grid = pushed_grid;
  *block = pushed_block;
  *lds = pushed_lds;
  *stream = pushed_stream;
  return 0;
}
int hipLaunchKernel(const void* f, Dim grid, Dim block, void**, size_t, void*) {
  launches().push_back({names()[f], grid, block});
  return 0;
}
int hipGetLastError(void) { return 0; }

void launches_clear(void) { launches().clear(); }
int launches_count(void) { return static_cast<int>(launches().size()); }
// name, and {grid x, y, z, block x, y, z} of launch i
const char* launches_get(int i, uint32_t* out) {
  const Launch& l = launches()[i];
  out[0] = l.grid.x, out[1] = l.grid.y, out[2] = l.grid.z;
  out[3] = l.block.x, out[4] = l.block.y, out[5] = l.block.z;
  return l.name.c_str();
}
}
