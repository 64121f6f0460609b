// The HIP calls that the library's host code makes, on the CPU: device memory is
// host memory that no kernel touches, and launches are noted down and not run.
// Loaded before the library with its symbols global, so that they are found first.
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <vector>

namespace {

struct Dim {
    uint32_t x, y, z;
};

struct Launch {
    const void *fn;
    uint32_t grid[3], block[3];
    uint64_t lds;
};
std::vector<Launch> launches;

}  // namespace

extern "C" {

int hipGetDevice(int *device)
{
    *device = 0;
    return 0;
}
int hipSetDevice(int) { return 0; }
int hipMalloc(void **p, size_t bytes)
{
    *p = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
    return *p ? 0 : 2;
}
int hipFree(void *p)
{
    std::free(p);
    return 0;
}
int hipMemcpy(void *to, const void *from, size_t bytes, int)
{
    std::memcpy(to, from, bytes);
    return 0;
}
int hipFuncSetAttribute(const void *fn, int, int) { return fn ? 0 : 1; }
int hipGetLastError() { return 0; }
int hipLaunchKernel(const void *fn, Dim grid, Dim block, void **, size_t lds, void *)
{
    launches.push_back({fn, {grid.x, grid.y, grid.z}, {block.x, block.y, block.z}, lds});
    return 0;
}

// The launches since the last call, up to n of them, into out.
int stub_launches(Launch *out, int n)
{
    const int held = (int)launches.size();
    for (int i = 0; i < held && i < n; i++)
        out[i] = launches[i];
    launches.clear();
    return held;
}

}  // extern "C"
