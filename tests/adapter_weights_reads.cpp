// Host program of test_adapter_weights_reads.py: the loads of an adapter's weights, lane by lane, from memory whose last element is the last one of
// the adapter's own rank and behind which there is none (a page without access).  Exit code 0: every value as it has to be, and nothing else read.
#include <sys/mman.h>

#include <cstdio>
#include <cstring>

#include "../paper_1805_10692_amd/csrc/adapter_weights.hpp"

using namespace cer;

template <class TW, bool kAlong>
int check(const char* name) {
    constexpr size_t kBytes = 1 << 20, kPage = 4096;
    char* room = static_cast<char*>(mmap(nullptr, kBytes + kPage, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    if (room == MAP_FAILED || mprotect(room + kBytes, kPage, PROT_NONE)) return 2;
    for (int rank = 1; rank <= 72; ++rank)
        for (int ld : {kAlong ? 64 : rank, kAlong ? 77 : 75}) {
            const int64_t numbers = kAlong ? (int64_t)(rank - 1) * ld + 64 : 63 * (int64_t)ld + rank;
            TW* w = reinterpret_cast<TW*>(room + kBytes) - numbers;
            for (int o = 0; o < 64; ++o)
                for (int r = 0; r < rank; ++r) w[kAlong ? r * ld + o : o * ld + r] = (TW)(float)((o * 3 + r * 7) % 61 + 1);
            for (int r0 = 0; r0 < 96; r0 += 32)
                for (int lane = 0; lane < 64; ++lane) {
                    const int i = lane % 16, low = r0 + lane / 16 * 8;
                    std::printf("%s rank %d ld %d ranks from %d lane %d\r", name, rank, ld, r0, lane);
                    Vec<TW, 8> u[4];
                    weights_of<TW, kAlong>(w, (uint32_t)(kAlong ? 4 * i : 4 * i * ld) * sizeof(TW), ld, rank, low, u);
                    for (int j = 0; j < 4; ++j)
                        for (int e = 0; e < 8; ++e) {
                            const float want = low + e < rank ? ((4 * i + j) * 3 + (low + e) * 7) % 61 + 1 : 0;
                            if ((float)u[j][e] != want) {
                                std::printf("\n%g is not %g\n", (double)u[j][e], (double)want);
                                return 1;
                            }
                        }
                }
        }
    return 0;
}

int main() {
    setvbuf(stdout, nullptr, _IONBF, 0);
    if (int e = check<float, true>("float rows")) return e;
    if (int e = check<float, false>("float")) return e;
    if (int e = check<__bf16, true>("bf16 rows")) return e;
    if (int e = check<__bf16, false>("bf16")) return e;
    if (int e = check<_Float16, true>("fp16 rows")) return e;
    if (int e = check<_Float16, false>("fp16")) return e;
    std::printf("\ndone\n");
    return 0;
}
