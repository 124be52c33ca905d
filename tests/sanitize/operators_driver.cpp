// Host sanitizer driver for the operators without a context: their translation units, compiled with -fsanitize=address,undefined on the host side,
// through work space sizes and argument checks at the ends of the integers, and, where there is no GPU to launch on, through the choice of kernels
// and the sizes of launches up to the error that the launch returns.  Structures and tables are exactly sized.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <memory>
#include <vector>

#include <hip/hip_runtime.h>

#include "bagel.h"

#define EXPECT(cond)                                                                       \
    do {                                                                                   \
        if (!(cond)) {                                                                     \
            std::printf("operators sanitizer driver: FAILED at line %d: %s (%s)\n", __LINE__, #cond, bagel_last_error(nullptr)); \
            return 1;                                                                      \
        }                                                                                  \
    } while (0)

static const int64_t MOST64 = std::numeric_limits<int64_t>::max(), LEAST64 = std::numeric_limits<int64_t>::min();
static const int32_t MOST32 = std::numeric_limits<int32_t>::max(), LEAST32 = std::numeric_limits<int32_t>::min();
static void *const P = reinterpret_cast<void *>(0x100000);       // never read or written here

static bagel_join join(int64_t rows, int32_t width, int dtype)
{
    bagel_join j;
    std::memset(&j, 0, sizeof(j));
    j.rows = rows; j.width = width; j.dtype = dtype; j.act = BAGEL_ACT_SILU; j.eps = 1e-6f;
    for (bagel_matrix *m : {&j.branch, &j.gate, &j.resid, &j.out, &j.normed, &j.d_out, &j.d_normed, &j.d_branch, &j.d_gate, &j.d_resid}) *m = {P, width};
    j.d_scale = j.d_post_weight = j.d_pre_weight = (float *)P;
    j.workspace = P; j.workspace_bytes = MOST64;
    return j;
}

static bagel_gated_recurrence recurrence(int64_t rows, int32_t width, int dtype, int32_t sequences, bool offsets)
{
    bagel_gated_recurrence r;
    std::memset(&r, 0, sizeof(r));
    r.rows = rows; r.width = width; r.dtype = dtype; r.sequences = sequences; r.offsets = offsets ? (const int32_t *)P : nullptr;
    for (bagel_matrix *m : {&r.value, &r.forget, &r.hidden, &r.d_hidden, &r.d_value, &r.d_forget}) *m = {P, width};
    r.carry = r.state = r.d_bias = (float *)P;
    r.workspace = P; r.workspace_bytes = MOST64;
    return r;
}

int main()
{
    int devices = 0;
    const bool launches = hipGetDeviceCount(&devices) != hipSuccess || devices == 0;
    (void)hipGetLastError();
    const int refused = BAGEL_EINVAL, failed = BAGEL_EHIP;
    const int idle = hipGetLastError() == hipSuccess ? BAGEL_OK : failed;      // of a pass without work: without a GPU that question is an error itself

    for (int64_t rows : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)MOST32, (int64_t)1 << 31, MOST64})
        for (int32_t width : {LEAST32, -1, 0, 1, 64, 16384, 16385, (1 << 20) - 1, 1 << 20, MOST32}) {
            const int64_t a = bagel_block_join_workspace(rows, width), b = bagel_recurrence_workspace(rows, width);
            EXPECT(rows < 0 || width < 1 || width > BAGEL_JOIN_MAX_WIDTH ? a == refused : a >= 0);
            EXPECT(rows < 0 || rows > MOST32 || width < 1 || width >= 1 << 20 ? b == refused : b > 0);
            EXPECT(rows < 0 || rows > MOST32 ? bagel_recurrence_carry_rows(rows) == refused : bagel_recurrence_carry_rows(rows) == (rows + 127) / 128);
        }

    // every tile, types and sizes at their ends; a launch without a GPU fails, and what does not launch is refused or has nothing to do
    for (int dtype : {-1, BAGEL_FLOAT32, BAGEL_BFLOAT16, BAGEL_FLOAT16, 3})
        for (int32_t width : {LEAST32, 0, 1, 3, 7, 8, 64, 100, 128, 256, 500, 512, 1000, 1024, 1280, 1500, 2048, 2500, 4000, 4096, 6000, 8192, 8193, 16384, 16385, MOST32})
            for (int64_t rows : {LEAST64, (int64_t)0, (int64_t)1, (int64_t)5000, ((int64_t)1 << 40) - 1, (int64_t)1 << 40, MOST64}) {
                const bool bad = dtype < 0 || dtype > 2 || width < 1 || width > BAGEL_JOIN_MAX_WIDTH || rows < 0 || rows >= (int64_t)1 << 40;
                auto j = std::make_unique<bagel_join>(join(rows, width, dtype));
                if (bad || rows == 0 || launches) EXPECT(bagel_block_join(j.get(), nullptr) == (bad ? refused : rows == 0 ? BAGEL_OK : failed));
                if (bad || launches) EXPECT(bagel_block_join_grad(j.get(), nullptr) == (bad ? refused : failed));
            }
    for (int64_t stride : {LEAST64, (int64_t)-1, (int64_t)63, (int64_t)1 << 40, MOST64}) {
        auto j = std::make_unique<bagel_join>(join(2, 64, 0));
        j->resid.stride = stride;
        EXPECT(bagel_block_join(j.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "stride"));
    }
    for (int64_t bytes : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)15}) {
        auto j = std::make_unique<bagel_join>(join(2, 64, 0));
        j->workspace_bytes = bytes;
        EXPECT(bagel_block_join_grad(j.get(), nullptr) == refused);
    }

    for (int dtype : {-1, BAGEL_FLOAT32, BAGEL_BFLOAT16, BAGEL_FLOAT16})
        for (int32_t width : {LEAST32, 0, 1, 2, 64, 65, 256, 777, 1024, (1 << 20) - 1, 1 << 20, MOST32})
            for (int64_t rows : {LEAST64, (int64_t)0, (int64_t)1, (int64_t)129, (int64_t)8200, ((int64_t)1 << 29) - 1, (int64_t)MOST32, MOST64})
                for (int32_t sequences : {LEAST32, 0, 1, 3, (1 << 28) - 1, MOST32})
                    for (bool offsets : {false, true}) {
                        auto r = std::make_unique<bagel_gated_recurrence>(recurrence(rows, width, dtype, sequences, offsets));
                        const bool sizes = dtype < 0 || width < 1 || width >= 1 << 20 || rows < 0 || rows > MOST32 || sequences < 0;
                        const bool bad = sizes || rows * ((width + 63) / 64) >= (int64_t)1 << 29 || sequences >= 1 << 28 || (rows > 0 && sequences == 0) ||
                                         (rows > 0 && !offsets && rows % sequences != 0);
                        if (bad || launches) {
                            EXPECT(bagel_recurrence(r.get(), nullptr) == (bad ? refused : rows == 0 ? idle : failed));
                            EXPECT(bagel_recurrence_grad(r.get(), nullptr) == (bad ? refused : failed));
                            r->final_state = r->d_initial = (float *)P;
                            const int64_t work = rows > 0 || sequences > 0;
                            EXPECT(bagel_recurrence(r.get(), nullptr) == (bad ? refused : work ? failed : idle));
                        }
                        const bool step = sizes || (int64_t)sequences * width >= (int64_t)1 << 38;
                        if (step || sequences == 0 || launches)
                            EXPECT(bagel_recurrence_step(r.get(), nullptr) == (step ? refused : sequences == 0 ? BAGEL_OK : failed));
                    }

    // updates: many tensors, sizes at their ends
    for (int bits : {8, 32})
        for (int64_t count : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)5'000'000, ((int64_t)1 << 38) - 1, (int64_t)1 << 38, MOST64})
            for (int32_t n : {1, 47, 48, 49, 200})
                for (int draws : {-1, BAGEL_DRAWS_MIXED, BAGEL_DRAWS_GIVEN, 2})
                    for (int64_t step : {LEAST64, (int64_t)0, (int64_t)1, MOST64}) {
                        std::vector<bagel_adamw_tensor> t(n);
                        for (auto &x : t) x = {(float *)P, P, P, P, (float *)P, (float *)P, P, count, 0.01};
                        bagel_adamw o;
                        std::memset(&o, 0, sizeof(o));
                        o.step = step; o.lr = 1e-3; o.beta1 = 0.9; o.beta2 = 0.999; o.eps = 1e-8; o.state_bits = bits; o.seed = 0xFFFFFFFFu; o.draws = draws;
                        const bool bad = count < 0 || count >= (int64_t)1 << 38 || draws < 0 || draws > 1 || step < 1;
                        if (bad || count == 0 || launches) EXPECT(bagel_adamw_step(t.data(), n, &o, nullptr) == (bad ? refused : count == 0 ? BAGEL_OK : failed));
                    }
    std::printf("operators sanitizer driver: ok%s\n", launches ? "" : ", without launches (there is a GPU)");
    return 0;
}
