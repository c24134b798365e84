// A stand-in for the HIP runtime in tests without a GPU: it keeps a record of what the library asks for and does none of it.
// Device addresses are numbers that nothing is stored at.
#include <unistd.h>

#include <cstdio>
#include <cstring>
#include <map>
#include <mutex>
#include <string>
#include <vector>

struct Dim3 {
  unsigned x, y, z;
};
struct Call {
  Dim3 grid, block;
  size_t lds;
  void* stream;
};

static std::mutex mu;
static std::vector<std::string> record;
static std::map<const void*, std::string>& kernels() {
  static std::map<const void*, std::string> names;
  return names;
}
static unsigned delay_us = 0;
static size_t next_address = (size_t)1 << 40;
static thread_local Call pushed;

template <class... A>
static void note(const char* fmt, A... a) {
  char line[512];
  snprintf(line, sizeof line, fmt, a...);
  std::lock_guard<std::mutex> lock(mu);
  record.push_back(std::to_string(gettid()) + " " + line);
}

extern "C" {

void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { kernels()[host] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream) {
  pushed = {grid, block, lds, stream};
  return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
  *grid = pushed.grid, *block = pushed.block, *lds = pushed.lds, *stream = pushed.stream;
  return 0;
}
int hipLaunchKernel(const void* host, Dim3 grid, Dim3 block, void**, size_t lds, void* stream) {
  if (delay_us) usleep(delay_us);
  note("launch %s %u %u %u %u %zu %zu", kernels()[host].c_str(), grid.x, grid.y, grid.z, block.x, lds, (size_t)stream);
  return 0;
}
int hipMalloc(void** p, size_t bytes) {
  {
    std::lock_guard<std::mutex> lock(mu);
    *p = (void*)next_address;
    next_address += (bytes + 4095) / 4096 * 4096 + 4096;
  }
  note("malloc %zu %zu", bytes, (size_t)*p);
  return 0;
}
int hipFree(void* p) {
  note("free %zu", (size_t)p);
  return 0;
}
int hipStreamSynchronize(void* stream) {
  note("wait %zu", (size_t)stream);
  return 0;
}
int hipDeviceGetAttribute(int* v, int, int) {
  *v = 256;            // compute units
  return 0;
}
int hipGetDevice(int* d) {
  *d = 0;
  return 0;
}
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipGetLastError(void) { return 0; }
const char* hipGetErrorString(int) { return "?"; }
int hipGetSymbolAddress(void** p, const void*) {
  *p = (void*)((size_t)1 << 39);
  return 0;
}
int hipEventCreate(void** e) {
  *e = nullptr;
  return 0;
}
int hipEventDestroy(void*) { return 0; }
int hipEventRecord(void*, void*) { return 0; }
int hipEventSynchronize(void*) { return 0; }
int hipEventElapsedTime(float* ms, void*, void*) {
  *ms = 0.f;
  return 0;
}

// for the tests
void fake_delay(unsigned us) { delay_us = us; }
size_t fake_take(char* out, size_t room) {        // the record as lines; emptied if there was room for it
  std::lock_guard<std::mutex> lock(mu);
  std::string all;
  for (const std::string& s : record) all += s + "\n";
  if (all.size() + 1 <= room) {
    memcpy(out, all.c_str(), all.size() + 1);
    record.clear();
  }
  return all.size() + 1;
}
}
