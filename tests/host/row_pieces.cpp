// The pieces of eight elements that the gradients of a gated pair take of dy, of tensors that end where the memory of this process does: a read behind the
// last element ends the program.  Prints "pieces <n> wrong <m>".
#include <sys/mman.h>
#include <unistd.h>

#include <cstdint>
#include <cstdio>

#include "../../paper_2304_07741_amd/csrc/product_kernels.hpp"
#include "../../paper_2304_07741_amd/csrc/row_util.hpp"

static long g_pieces = 0, g_wrong = 0;

template <class T>
static void look(bool f32, char* end, int64_t rows, int64_t width) {
    T* at = reinterpret_cast<T*>(end) - rows * width;
    for (int64_t k = 0; k < rows * width; k++) at[k] = (T)(k % 1000 + 1);
    for (int64_t r = 0; r < rows; r++)
        for (int64_t col = 0; col < canvas::product::padded(f32, width); col += 8) {
            T v[8];
            canvas::rows::load8(at + r * width, col, width, v);
            for (int e = 0; e < 8; e++) g_wrong += v[e] != (col + e < width ? (T)((r * width + col + e) % 1000 + 1) : (T)0);
            g_pieces++;
        }
}

int main() {
    const size_t page = (size_t)sysconf(_SC_PAGESIZE), bytes = 64 * page;
    char* base = static_cast<char*>(mmap(nullptr, bytes + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    if (base == MAP_FAILED || mprotect(base + bytes, page, PROT_NONE)) return 2;
    for (int64_t width = 1; width <= 200; width++)  // every remainder by 16
        for (int64_t rows : {1, 2, 128}) {
            look<float>(true, base + bytes, rows, width);
            look<uint16_t>(false, base + bytes, rows, width);
        }
    printf("pieces %ld wrong %ld\n", g_pieces, g_wrong);
    return 0;
}
