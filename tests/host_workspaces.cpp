// The device memory that the library allocates over a list of calls: the double
// of the HIP runtime in host_launches.cpp with its hipMalloc counted.
//
//   host_workspaces LIB < commands
//
// Takes host_launches' commands of one call each; prints "STATUS ALLOCATIONS
// BYTES LARGEST" after every one: all so far, the largest allocation among them.
// A first line "memory BYTES" makes allocations that would leave less than
// nothing of that fail.
#define hipMalloc unbounded_malloc
#define main launches_main
#include "host_launches.cpp"
#undef hipMalloc
#undef main

namespace {
size_t g_allocations = 0, g_bytes = 0, g_largest = 0, g_memory = ~(size_t)0;
}

extern "C" int hipMalloc(void** p, size_t bytes) {
    if (bytes > g_memory - g_bytes) return t_error = 2;   // out of memory
    const int e = unbounded_malloc(p, bytes);
    if (e != 0) return e;
    ++g_allocations;
    g_bytes += bytes;
    if (bytes > g_largest) g_largest = bytes;
    return 0;
}

int main(int argc, char** argv) {
    if (argc != 2 || (g_lib = dlopen(argv[1], RTLD_NOW)) == nullptr) return 2;
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        if (line.rfind("memory ", 0) == 0) {
            std::string word;
            in >> word >> g_memory;
            continue;
        }
        Call c;
        if (!parse(in, c)) return 2;
        g_capturing = c.capturing;
        printf("%d", c.run());
        printf(" %zu %zu %zu\n", g_allocations, g_bytes, g_largest);
    }
    return 0;
}
