// The argument checks of the language-model operators (bns_lm_validate.hpp, plain C++) under the sanitizers: every combination of extreme values in their
// descriptions, and the overlap test against what it means, byte by byte, for small matrices.
#include <stdio.h>

#include <vector>

#include "../../paper_1810_10962_amd/csrc/bns_lm_validate.hpp"

using namespace bns;

static int64_t accepted = 0, rejected = 0;

static void count(bns_status s) { ++(s == BNS_OK ? accepted : rejected); }

static void extremes() {
    const int64_t rows[] = {INT64_MIN, -1, 0, 1, 7, (int64_t(1) << 20), (int64_t(1) << 20) + 1, (int64_t(1) << 31) - 1, int64_t(1) << 31, INT64_MAX};
    const int32_t sizes[] = {INT32_MIN, -1, 0, 1, 64, 1001, 16384, 16385, 65536, 65537, (1 << 24) - 1, 1 << 24, (1 << 30) - 1, 1 << 30, INT32_MAX};
    const int64_t strides[] = {INT64_MIN, -1, 0, 1, 1001, 65536, (int64_t(1) << 31) - 1, int64_t(1) << 31, INT64_MAX};
    const int32_t small[] = {INT32_MIN, -1, 0, 1, 2, 32, 64, 96, 128, INT32_MAX};
    const float reals[] = {-1.f, -0.f, 0.f, 1e-6f, 1.f, __builtin_inff(), __builtin_nanf("")};
    for (int64_t r : rows)
        for (int32_t w : sizes)
            for (int64_t s : strides) {
                for (int32_t v : sizes)
                    for (int32_t e : {-1, 0, 1, 2}) {
                        HeadDims hd;
                        const bns_head h = {r, s, s, w, v, e, v};
                        count(check_head(&h, &hd));
                        for (float f : reals) {
                            DistillDims dd;
                            const bns_distill d = {r, s, 0, v, w, e, f};
                            const bns_status st = check_distill(&d, &dd);
                            count(st);
                            if (st == BNS_OK) {     // the byte counts of accepted descriptions do not wrap
                                const Matrix m = matrix(&dd, dd.tokens, dd.vocab, dd.logits_stride, 4);
                                if (dd.tokens > 0 && m.bytes / 4 < size_t(dd.vocab)) __builtin_trap();
                            }
                        }
                    }
                for (int32_t g : small)
                    for (int32_t o : {-1, 0, 1, 2})
                        for (float f : reals) {
                            RmsDims d;
                            const bns_rms m = {r, s, 0, s, 0, w, 1, 0, o, g, o, f};
                            const bns_status st = check_rms(&m, &d);
                            count(st);
                            if (st == BNS_OK && (d.groups < 1 || d.x_stride < d.width)) __builtin_trap();
                        }
            }
    RmsDims rd;
    HeadDims hd;
    DistillDims dd;
    count(check_rms(nullptr, &rd));
    count(check_head(nullptr, &hd));
    count(check_distill(nullptr, &dd));
    printf("accepted %lld rejected %lld\n", static_cast<long long>(accepted), static_cast<long long>(rejected));
}

// Matrices of bytes in one buffer: collide() never lets a shared byte pass (except in place), and lets interleaved halves pass.
static void overlaps() {
    static char buffer[512];
    long checked = 0, apart = 0;
    for (int rows = 1; rows <= 4; ++rows)
        for (int wa = 1; wa <= 6; ++wa)
            for (int wb = 1; wb <= 6; ++wb)
                for (int sa = wa; sa <= 12; ++sa)
                    for (int sb = wb; sb <= 12; ++sb)
                        for (int at = 0; at < 40; ++at) {
                            const Matrix a = matrix(buffer + 100, rows, wa, sa, 1), b = matrix(buffer + 80 + at, rows, wb, sb, 1);
                            std::vector<char> used(512, 0);
                            for (int r = 0; r < rows; ++r)
                                for (int c = 0; c < wa; ++c) used[size_t(100 + r * sa + c)] = 1;
                            bool shared = false;
                            for (int r = 0; r < rows; ++r)
                                for (int c = 0; c < wb; ++c) shared |= used[size_t(80 + at + r * sb + c)] != 0;
                            const bool refused = collide(a, b, false, size_t(wa), size_t(wb));
                            if (shared && !refused) __builtin_trap();
                            if (!refused) ++apart;
                            if (collide(a, b, true, size_t(wa), size_t(wb)) && !refused) __builtin_trap();
                            ++checked;
                        }
    const Matrix left = matrix(buffer, 4, 8, 16, 1), right = matrix(buffer + 8, 4, 8, 16, 1), none = matrix(nullptr, 4, 8, 16, 1), empty = matrix(buffer, 0, 8, 16, 1);
    if (collide(left, right, false, 8, 8) || collide(right, left, false, 8, 8)) __builtin_trap();
    if (collide(left, none, false, 8, 8) || collide(left, empty, false, 8, 8) || collide(left, left, true, 8, 8) || !collide(left, left, false, 8, 8)) __builtin_trap();
    printf("checked %ld apart %ld\n", checked, apart);
}

int main(int argc, char**) {
    if (argc > 1) overlaps();
    else extremes();
    return 0;
}
