// Stands in front of the HIP runtime's kernel launch (LD_PRELOAD) and writes down what a call launches, instead of launching it: for tests without a GPU.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <map>
#include <string>

namespace {
struct Dim3 {
    uint32_t x, y, z;
};
std::map<const void*, std::string>& names() {
    static std::map<const void*, std::string> m;
    return m;
}
std::string text;
int head = 0;  // bytes of a kernel's first argument that are written down
}  // namespace

extern "C" {

void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) {
    names()[host] = name;  // (not passed on: nothing is launched)
}

// (the launch's configuration, which the runtime refuses to hold without a GPU)
static Dim3 conf[2];
static size_t conf_lds;
static void* conf_stream;
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void* stream) {
    conf[0] = grid;
    conf[1] = block;
    conf_lds = lds;
    conf_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
    *grid = conf[0];
    *block = conf[1];
    *lds = conf_lds;
    *stream = conf_stream;
    return 0;
}
int hipGetLastError() { return 0; }

int hipLaunchKernel(const void* host, Dim3 grid, Dim3 block, void** args, size_t, void*) {
    char line[160];
    snprintf(line, sizeof line, " %u %u %u %u %u %u ", grid.x, grid.y, grid.z, block.x, block.y, block.z);
    text += names()[host] + line;
    for (int i = 0; i < head; ++i) {
        snprintf(line, sizeof line, "%02x", reinterpret_cast<const unsigned char*>(args[0])[i]);
        text += line;
    }
    text += '\n';
    return 0;
}

// What was launched since the last call of this: a line for each, the kernel's name, grid, block and the first `bytes` bytes of its first argument
// (of the launches that follow)
const char* launch_log(int bytes) {
    static std::string out;
    out.swap(text);
    text.clear();
    head = bytes;
    return out.c_str();
}

}  // extern "C"
