// Launches of the adapters' kernels as they leave the library's own launcher: the runtime's calls below are this program's, and look at each kernel's
// name, for what it was made, and at what its launch gives it.  Nothing runs on a GPU.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <map>
#include <string>

#include "../../include/fq.h"
#include "../../paper_2511_12653_amd/csrc/fq_adapters.h"

static int failures = 0, launches = 0, forms[2][5][5][9];
static long long shown[6];
#define CHECK(c) do { if (!(c) && ++failures < 40) std::printf("%s:%d: %s (%lld %lld %lld, %lld by %lld, type %lld)\n", __FILE__, __LINE__, #c, \
                                                                shown[0], shown[1], shown[2], shown[3], shown[4], shown[5]); } while (0)

static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> all;
    return all;
}

static struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} configured;

static long long ceiling(long long v, long long by) { return (v + by - 1) / by; }

extern "C" {

void **__hipRegisterFatBinary(const void *) { static void *one; return &one; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *function, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[function] = name; }

hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    configured = {grid, block, lds, stream};
    return hipSuccess;
}

hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = configured.grid; *block = configured.block; *lds = configured.lds; *stream = configured.stream;
    return hipSuccess;
}

hipError_t hipGetLastError() { return hipSuccess; }

hipError_t hipLaunchKernel(const void *function, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t)
{
    ++launches;
    const fq::AdapterArgs &a = *(const fq::AdapterArgs *)args[0];
    const std::string &name = names()[function];
    int n, tt, j, few, brief, nt, nr;
    CHECK(grid.y == 1 && grid.z == 1 && block.y == 1 && block.z == 1);
    if (name.find("adapter_group_kernel") != std::string::npos) {
        CHECK(block.x == 1024 && grid.x == 1 && lds >= (size_t)(a.count + 1) * 16 * sizeof(int) && a.count <= fq::kMostGrouped);
        return hipSuccess;
    }
    CHECK(block.x == 256);
    const char *numbers = std::strstr(name.c_str(), "Li");
    if (name.find("adapter_up_kernel") != std::string::npos) {
        if (!numbers || std::sscanf(numbers, "Li%dELi%dELi%dELb%dELb%dE", &n, &tt, &j, &few, &brief) != 5) return hipErrorInvalidValue;
        // two FP16 numbers for each place of a row of t (whole 32 ranks and 8 more) of each of the kernel's 16 tt tokens
        CHECK(lds >= (size_t)2 * 16 * tt * (ceiling(a.rank, 32) * 32 + 8) * 2);
        CHECK(lds + 6144 <= 160 * 1024);
        CHECK(grid.x == (unsigned)a.tiles_most * (unsigned)a.groups);
        CHECK(32 * j >= a.rank && (few || a.n >= n) && (tt == 1 || tt == 2 || (tt == 4 && j < 8)));
        CHECK(brief || a.rank >= 8);
        CHECK(!brief || a.rank < 8 || few);
        CHECK(!brief || few || a.n * a.rank >= 8 || a.count == 0);
        ++forms[brief][n][tt][j];
    } else {
        CHECK(a.count > 0 && grid.x == (unsigned)a.tiles_most * (unsigned)a.splits * (unsigned)a.chunks);
        if (!numbers || std::sscanf(numbers, "Li%dELi%dE", &nt, &nr) != 2) return hipErrorInvalidValue;
        CHECK(16LL * nr * a.chunks >= a.rank);
        if (name.find("adapter_down_ring_kernel") != std::string::npos) {
            // rings of two slots at least, which later hold the sums of all four wavefronts
            const int size = a.x_type == FQ_F32 ? 4 : a.x_type == FQ_F16 ? 2 : 1;
            CHECK(a.x_bytes && lds >= (size_t)4 * 2 * (nt * size + nr * 2) * 1024 && lds >= (size_t)4 * nt * nr * 1024 && lds + 6144 <= 160 * 1024);
        } else {
            CHECK(name.find("adapter_down_kernel") != std::string::npos && lds == 0);
        }
    }
    return hipSuccess;
}

}  // extern "C"

static char *at(int i) { return (char *)(uintptr_t)((unsigned long long)i << 56); }

static unsigned long long state = 1;
static long long pick(long long most)
{
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    const int bits = (int)((state >> 40) % 63);
    const unsigned long long r = (state >> 20) ^ (state << 37);
    return (long long)(r & ((1ull << bits) - 1)) % (most + 1);
}

static void adapters(long long m, long long n, long long k, long long count, long long rank, int type)
{
    shown[0] = m; shown[1] = n; shown[2] = k; shown[3] = count; shown[4] = rank; shown[5] = type;
    fq_adapters d;
    std::memset(&d, 0, sizeof d);
    d.m = m; d.n = n; d.k = k; d.count = count; d.rank = rank;
    d.x_dtype = type % 3; d.y_dtype = type >> 2 & 1; d.base_dtype = type >> 3 & 1; d.xs_step = 1;
    d.ldx = k + (type >> 4 & 1); d.ldy = n; d.ldbase = n;
    d.x = at(1); d.xs = (float *)at(2); d.ids = (int32_t *)at(3); d.a = at(4) + (type >> 5 & 1) * 2; d.b = at(5); d.scale = (float *)at(6);
    d.base = type & 64 ? nullptr : at(7); d.y = at(8);
    const size_t bytes = fq_adapters_workspace_bytes(&d);
    CHECK(bytes > 0);
    CHECK(fq_adapters_forward(&d, at(9), bytes, nullptr) == FQ_OK);
}

int main()
{
    for (long long rank : {1LL, 2LL, 3LL, 4LL, 5LL, 6LL, 7LL, 8LL, 16LL, 33LL, 64LL, 65LL, 128LL, 129LL, 256LL})
        for (long long m : {1LL, 2LL, 16LL, 27LL, 48LL, 64LL, 65LL, 256LL, 512LL, 1000LL, 1023LL, 1024LL, 2000LL, 4096LL, 4097LL, 8192LL, 70000LL})
            for (long long n : {1LL, 2LL, 3LL, 4LL, 7LL, 64LL, 1000LL, 4096LL, 7953LL, 8192LL, 11008LL, 1LL << 20})
                for (long long k : {1LL, 8LL, 16LL, 512LL, 4096LL})
                    for (long long count : {1LL, 2LL, 8LL, 32LL, 64LL, 1024LL, 1025LL}) adapters(m, n, k, count, rank, (int)pick(127));
    for (int i = 0; i < 100000; ++i) adapters(pick(100000), pick(1LL << 20), pick(1LL << 20), pick(3000), pick(256), (int)pick(127));
    for (int brief = 0; brief < 2; ++brief)
        for (int n = 0; n < 5; ++n)
            for (int tt = 0; tt < 5; ++tt)
                for (int j = 0; j < 9; ++j)
                    if (forms[brief][n][tt][j]) std::printf("rank < 8: %d, channels %d, tokens %d, ranks up to %d: %d\n", brief, n, 16 * tt, 32 * j, forms[brief][n][tt][j]);
    std::printf("adapters: %d failures, %d launches\n", failures, launches);
    return failures != 0;
}
