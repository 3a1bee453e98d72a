// For every line "type N D V" of the input: the forms that a cross entropy and its gradients of these sizes take, one a line; for "q8 M K N": the
// form of a product in 8-bit integers.  A form whose ring of buffers a call never fills again is told apart ("short"); a line of its own ends each answer.
#include <cstdio>
#include <cstring>
#include <string>

#include "scd_lm_shape.h"

using namespace scd::lm;

static const char* name(LogitsTile t)
{
    const char* names[] = {"256", "128", "deep 128", "64", "64 tokens", "32 tokens"};
    return names[(int)t];
}

int main()
{
    char type[8];
    long a, b, c;
    while (std::scanf("%7s %ld %ld %ld", type, &a, &b, &c) == 4) {
        if (!std::strcmp(type, "q8")) {
            const char* names[] = {"few", "narrow", "256", "128", "64"};
            const Q8Form f = q8_form(a, b, c);
            std::printf("q8 %s", names[(int)f]);
            if (f == Q8Form::few) std::printf(" own %d", q8_few_owns(a, b));
            else std::printf("%s", q8_stride(b) / kTileStep < 8 ? " short" : "");
            std::printf("\n--\n");
            continue;
        }
        const int dt = !std::strcmp(type, "f32") ? SCD_REAL_F32 : !std::strcmp(type, "f16") ? SCD_REAL_F16 : SCD_REAL_BF16;
        const Shape s = shape_of(dt, a, b, c);
        const std::string t = s.f32 && !s.split ? "f32 as it is" : type;
        const char* lost = cdiv(s.ld * s.bytes, kTileStep) < 8 ? " short" : "";
        const char* copied = s.copies_w ? s.piece < s.V ? " copied in pieces" : " copied" : "";
        if (s.z_splits > 1) {
            std::printf("%s logits in shares, %s%s\n", t.c_str(), takes_few(s.N, s.V) ? s.N <= 32 ? "32 tokens" : "64 tokens" : "64", copied);
        } else {
            const int64_t forward = s.copies_w ? s.piece : s.V;
            std::printf("%s loss %s%s%s\n", t.c_str(), name(logits_tile(s, forward, s.N)), copied, lost);
            for (int64_t v0 = 0; v0 < s.V; v0 += s.piece) {
                const int64_t width = s.V - v0 < s.piece ? s.V - v0 : s.piece;
                std::printf("%s dz %s%s%s\n", t.c_str(), name(logits_tile(s, width, s.N)), v0 ? ", later piece" : "", lost);
            }
        }
        const std::string grads = s.grads ? std::to_string(s.grads) : s.N <= 32 ? "32 tokens" : "64 tokens";
        const char *pieces = s.piece < s.V ? ", pieces" : "", *planes = s.dz_planes == 2 ? ", two planes" : "";
        std::printf("%s dX %s%s%s%s\n", t.c_str(), grads.c_str(), planes, s.splits > 1 ? ", shares" : "", pieces);
        const char* width = dw_walks(s, s.piece, true) ? "walks" : grads.c_str();
        std::printf("%s dW %s%s%s%s%s\n", t.c_str(), width, planes, s.w_splits > 1 ? ", shares" : "", pieces, s.grads == 256 && cdiv(s.N, 64) < 8 ? " short" : "");
        std::printf("--\n");
    }
    return 0;
}
