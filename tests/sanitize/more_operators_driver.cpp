// Host sanitizer driver for layer norm, linear attention and the clipping of gradients: their translation units, compiled with -fsanitize=address,undefined on
// the host side, through work space sizes and argument checks at the ends of the integers, and, where there is no GPU to launch on, through the choice of
// kernels and the sizes of launches up to the error that the launch returns.  Structures and tables are exactly sized.
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
            std::printf("more operators sanitizer driver: FAILED at line %d: %s (%s)\n", __LINE__, #cond, bagel_last_error(nullptr)); \
            return 1;                                                                      \
        }                                                                                  \
    } while (0)

static const int64_t MOST64 = std::numeric_limits<int64_t>::max(), LEAST64 = std::numeric_limits<int64_t>::min();
static const int32_t MOST32 = std::numeric_limits<int32_t>::max(), LEAST32 = std::numeric_limits<int32_t>::min();
static void *const P = reinterpret_cast<void *>(0x100000);       // never read or written here

static bagel_norm norm(int64_t rows, int32_t width, int32_t groups, int dtype)
{
    bagel_norm n;
    std::memset(&n, 0, sizeof(n));
    n.rows = rows; n.width = width; n.groups = groups; n.dtype = dtype; n.eps = 1e-6f;
    for (bagel_matrix *m : {&n.x, &n.out, &n.d_out, &n.d_x}) *m = {P, width};
    n.d_weight = n.d_bias = (float *)P;
    n.workspace = P; n.workspace_bytes = MOST64;
    return n;
}

static bagel_attention attention(int64_t rows, int32_t sequences, int32_t heads, int32_t states, int32_t dk, int32_t dv, int dtype, bool offsets)
{
    bagel_attention b;
    std::memset(&b, 0, sizeof(b));
    b.rows = rows; b.sequences = sequences; b.heads = heads; b.states = states; b.key_width = dk; b.value_width = dv; b.dtype = dtype; b.scale = 0.5f;
    b.offsets = offsets ? (const int32_t *)P : nullptr;
    b.log_decay = (const float *)P;
    const int64_t h = heads > 0 ? heads : 1, s = states > 0 ? states : 1, k = dk > 0 ? dk : 1, v = dv > 0 ? dv : 1;
    b.query = b.d_query = {P, h * k, k};
    b.key = b.d_key = {P, s * k, k};
    b.value = b.d_value = {P, s * v, v};
    b.out = b.d_out = {P, h * v, v};
    b.state = (float *)P;
    b.workspace = P; b.workspace_bytes = MOST64;
    return b;
}

int main()
{
    int devices = 0;
    const bool launches = hipGetDeviceCount(&devices) != hipSuccess || devices == 0;
    (void)hipGetLastError();
    const int refused = BAGEL_EINVAL, failed = BAGEL_EHIP;

    for (int dtype : {-1, BAGEL_FLOAT32, BAGEL_BFLOAT16, BAGEL_FLOAT16, 3})
        for (int32_t width : {LEAST32, -1, 0, 1, 3, 7, 8, 64, 100, 512, 1000, 1024, 2048, 4096, 8192, 16384, 16385, MOST32})
            for (int32_t groups : {LEAST32, -1, 0, 1, 2, 8, 25, 1024, 16384, MOST32})
                for (int64_t rows : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)5000, ((int64_t)1 << 40) - 1, (int64_t)1 << 40, MOST64}) {
                    const bool sizes = width < 1 || width > BAGEL_NORM_MAX_WIDTH || groups < 1 || width % groups != 0 || rows < 0 || rows >= (int64_t)1 << 40;
                    const bool bad = sizes || dtype < 0 || dtype > 2;
                    const int64_t bytes = bagel_layer_norm_workspace(rows, width, groups);
                    EXPECT(sizes ? bytes == refused : bytes >= 0 && bytes < (int64_t)1 << 31);
                    auto n = std::make_unique<bagel_norm>(norm(rows, width, groups, dtype));
                    if (bad || rows == 0 || launches) EXPECT(bagel_layer_norm(n.get(), nullptr) == (bad ? refused : rows == 0 ? BAGEL_OK : failed));
                    if (bad || launches) EXPECT(bagel_layer_norm_grad(n.get(), nullptr) == (bad ? refused : failed));
                    if (bytes <= 0 || bad) continue;
                    n->workspace_bytes = bytes - 1;
                    EXPECT(bagel_layer_norm_grad(n.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "too small"));
                }
    for (int64_t stride : {LEAST64, (int64_t)-1, (int64_t)63, (int64_t)1 << 40, MOST64}) {
        auto n = std::make_unique<bagel_norm>(norm(2, 64, 2, 0));
        n->x.stride = stride;
        EXPECT(bagel_layer_norm(n.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "stride"));
    }

    for (int dtype : {-1, BAGEL_FLOAT32, BAGEL_BFLOAT16, BAGEL_FLOAT16})
        for (int32_t dk : {LEAST32, 0, 1, 3, 8, 64, 65, 128, 129, MOST32})
            for (int32_t dv : {0, 1, 7, 64, 77, 128, MOST32})
                for (int64_t rows : {LEAST64, (int64_t)0, (int64_t)1, (int64_t)129, (int64_t)100'000, ((int64_t)1 << 28) - 1, (int64_t)1 << 28, MOST64})
                    for (int32_t sequences : {LEAST32, 0, 1, 3, (1 << 28) - 1, 1 << 28, MOST32})
                        for (int32_t states : {LEAST32, 0, 1, 2, 4096, MOST32})
                            for (bool offsets : {false, true}) {
                                const int32_t heads = states == 2 ? 4 : states;
                                auto b = std::make_unique<bagel_attention>(attention(rows, sequences, heads, states, dk, dv, dtype, offsets));
                                const bool sizes = rows < 0 || rows >= 1 << 28 || sequences < 0 || sequences >= 1 << 28 || states < 1 || heads > 4096 || dk < 1 || dk > 128 ||
                                                   dv < 1 || dv > 128 || (rows + sequences) * states >= (int64_t)1 << 31;
                                const bool inputs = sizes || dtype < 0;
                                const bool bad = inputs || (rows > 0 && (sequences == 0 || (!offsets && rows % sequences != 0)));
                                const int64_t bytes = bagel_linear_attention_workspace(b.get(), 0), back = bagel_linear_attention_workspace(b.get(), 1);
                                EXPECT(sizes ? bytes == refused && back == refused : bytes >= 0 && back == 2 * bytes);
                                const bool idles = rows == 0 && sequences == 0;
                                if (bad || launches) {
                                    EXPECT(bagel_linear_attention(b.get(), nullptr) == (bad ? refused : idles ? BAGEL_OK : failed));
                                    EXPECT(bagel_linear_attention_grad(b.get(), nullptr) == (bad ? refused : idles ? BAGEL_OK : failed));
                                }
                                const bool step = inputs || rows != sequences;
                                if (step || rows == 0 || launches) EXPECT(bagel_linear_attention_step(b.get(), nullptr) == (step ? refused : rows == 0 ? BAGEL_OK : failed));
                                if (bad || bytes <= 0) continue;
                                b->workspace_bytes = bytes - 1;
                                EXPECT(bagel_linear_attention(b.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "too small"));
                                b->workspace_bytes = back - 1;
                                EXPECT(bagel_linear_attention_grad(b.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "too small"));
                                b->workspace = nullptr;
                                EXPECT(bagel_linear_attention(b.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "needed"));
                            }
    // distances that a result's rows or heads overlap with, or that cannot be addressed
    for (int64_t rows : {(int64_t)2, ((int64_t)1 << 28) - 1})
        for (int64_t stride : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)63, (int64_t)127, (int64_t)1 << 40, MOST64})
            for (int64_t head : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)63, (int64_t)64, (int64_t)1 << 40, MOST64}) {
                auto b = std::make_unique<bagel_attention>(attention(rows, 1, 2, 2, 64, 64, 0, true));
                b->out = {P, stride, head};
                EXPECT(bagel_linear_attention(b.get(), nullptr) == refused);
            }
    for (int64_t stride : {((int64_t)1 << 33) + 1, ((int64_t)1 << 40) - 1})
        for (bagel_heads bagel_attention::*h : {&bagel_attention::query, &bagel_attention::key, &bagel_attention::value, &bagel_attention::out}) {
            auto b = std::make_unique<bagel_attention>(attention(((int64_t)1 << 28) - 1, 1, 2, 2, 64, 64, 0, true));
            (b.get()->*h).stride = stride;
            EXPECT(bagel_linear_attention(b.get(), nullptr) == refused && std::strstr(bagel_last_error(nullptr), "2^60"));
        }

    // many tensors of counts at their ends
    EXPECT(bagel_clip_norm_workspace(-1) == refused && bagel_clip_norm_workspace(LEAST32) == refused && bagel_clip_norm_workspace(0) > 0);
    for (int64_t count : {LEAST64, (int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)5'000'000, ((int64_t)1 << 38) - 1, (int64_t)1 << 38, MOST64})
        for (int32_t n : {0, 1, 95, 96, 97, 300})
            for (int32_t dtype : {-1, BAGEL_FLOAT32, BAGEL_BFLOAT16, BAGEL_FLOAT16, 3})
                for (bool written : {false, true}) {
                    std::vector<bagel_clip_tensor> t(n);
                    for (int32_t i = 0; i < n; ++i) {
                        void *const at = reinterpret_cast<void *>(((uintptr_t)i + 1) << 41);
                        t[i] = {at, written ? at : nullptr, count, dtype};
                    }
                    bagel_clip o;
                    std::memset(&o, 0, sizeof(o));
                    o.max_norm = 1.0f; o.eps = 1e-6f; o.norm = o.factor = (float *)P; o.workspace = P; o.workspace_bytes = MOST64;
                    const bool bad = n > 0 && (count < 0 || count >= (int64_t)1 << 38 || (count > 0 && (dtype < 0 || dtype > 2)));
                    if (bad || launches) EXPECT(bagel_clip_norm(t.data(), n, &o, nullptr) == (bad ? refused : failed));
                }
    // results in another tensor's place
    const auto overlapping = [&](int32_t n, int32_t which, uintptr_t out) {
        std::vector<bagel_clip_tensor> t(n);
        for (int32_t i = 0; i < n; ++i) t[i] = {reinterpret_cast<void *>((uintptr_t)(i + 1) << 20), reinterpret_cast<void *>((uintptr_t)(i + 1) << 20), 1000, BAGEL_FLOAT32};
        t[which].out = reinterpret_cast<void *>(out);
        bagel_clip o;
        std::memset(&o, 0, sizeof(o));
        o.max_norm = 1.0f; o.eps = 1e-6f; o.norm = o.factor = (float *)P; o.workspace = P; o.workspace_bytes = MOST64;
        const int r = bagel_clip_norm(t.data(), n, &o, nullptr);
        return r == refused && std::strstr(bagel_last_error(nullptr), "overlaps") ? 1 : r == failed ? 0 : -1;
    };
    if (launches)
        for (int32_t n : {2, 64, 65, 300}) {
            EXPECT(overlapping(n, 1, (uintptr_t)1 << 20) == 1);                          // the other's place
            EXPECT(overlapping(n, 1, ((uintptr_t)1 << 20) + 3996) == 1);                 // its last entry
            EXPECT(overlapping(n, 1, ((uintptr_t)2 << 20) + 4) == 1);                    // an entry on in its own
            EXPECT(overlapping(n, 1, ((uintptr_t)1 << 20) + 4000) == 0);                 // behind it
            EXPECT(overlapping(n, 1, (uintptr_t)2 << 20) == 0);
        }
    std::printf("more operators sanitizer driver: ok%s\n", launches ? "" : ", without launches (there is a GPU)");
    return 0;
}
