// Index arithmetic of windows and trees on the host: the line of the keys that rows see, and chains of parents, for good numbers and for wrong ones.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../../paper_2311_09549_amd/csrc/attention.h"

using namespace sck;

#define CHECK(x)                                                  \
    do {                                                          \
        if (!(x)) {                                               \
            printf("%s:%d: %s\n", __FILE__, __LINE__, #x);        \
            exit(1);                                              \
        }                                                         \
    } while (0)

// Every key that a row from position p on sees is in the line once, in order, in whole sixteens that hold one, and little else.
static void line_covers(int32_t length, int32_t window, int32_t sinks, int32_t p)
{
    const Span s = span_of(length, window, sinks, p);
    CHECK(s.first % 16 == 0 && s.skip % 16 == 0 && s.first >= 0 && s.skip >= 0 && s.length == length - s.skip);
    int64_t before = -1;
    std::vector<int> in(length, 0);
    for (int32_t v = 0; v < s.length; ++v) {
        const int32_t key = key_at(s, v);
        CHECK(key > before && key < length);
        before = key;
        in[key] = 1;
        if (v % 16 == 0) CHECK(key % 16 == 0);
    }
    const int32_t low = window_low(window, p);
    for (int32_t j = 0; j < length; ++j)
        if (j >= low || j < sinks) CHECK(in[j]);
    if (s.skip)   // a sixteen of the line has a key that is seen
        for (int32_t v = 0; v < s.length; v += 16) CHECK(key_at(s, v) + 15 >= low || key_at(s, v) < sinks);
    if (window > 0 && length > 0) CHECK(s.length <= 16 + 15 + (length - low) + (sinks < low ? sinks : low) || s.skip == 0);
}

int main()
{
    std::mt19937 rng(1);
    const auto pick = [&](std::vector<int64_t> special, int64_t most) { return (int32_t)(rng() % 2 ? special[rng() % special.size()] : rng() % (most + 1)); };
    for (int n = 0; n < 20000; ++n) {
        const int32_t length = pick({0, 1, 15, 16, 17, 127, 128, 129}, 600), p = length ? (int32_t)(rng() % (length + 3)) - 3 : -1;
        line_covers(length, pick({0, 1, 2, 15, 16, 17, 128, 1 << 30}, 600), pick({0, 1, 15, 16, 17, 1 << 30}, 300), p);
    }
    CHECK(window_low(1, -5) == 0 && window_low(1, 7) == 7 && window_low(8, 7) == 0 && window_low(0, 7) == 0 && window_low(1 << 30, (1 << 30) - 1) == 0);
    CHECK(span_of(1 << 30, 1, 1 << 30, (1 << 30) - 1).skip == 0);
    const Span far = span_of(1 << 30, 100, 5, (1 << 30) - 1);
    CHECK(far.first == 16 && key_at(far, far.length - 1) == (1 << 30) - 1 && far.length < 200);

    // chains: depths of good trees, and -1 from a wrong number on
    for (int n = 0; n < 2000; ++n) {
        const int count = 1 + rng() % 60;
        std::vector<int32_t> parent(count), depth(count);
        for (int i = 0; i < count; ++i) {
            parent[i] = (int32_t)(rng() % (i + 1)) - 1;
            depth[i] = parent[i] < 0 ? 0 : depth[parent[i]] + 1;
        }
        for (int i = 0; i < count; ++i) CHECK(depth_of(parent.data(), i) == depth[i]);
        const int wrong = rng() % count;
        const int32_t numbers[] = {-2, wrong, wrong + 1, INT32_MAX, INT32_MIN};
        parent[wrong] = numbers[rng() % 5];
        for (int i = 0; i < count; ++i) {
            bool below = false;
            for (int k = i; k >= 0 && !below; k = k == wrong ? -1 : parent[k]) below = k == wrong;
            CHECK(depth_of(parent.data(), i) == (below ? -1 : depth[i]));
        }
    }
    printf("ok\n");
    return 0;
}
