// The cosines and sines of rotary positions, plain or stretched over contexts longer than a model was trained on (host).
#include <cmath>

#include "lqq_common.h"

using namespace lqq;

extern "C" int attn_rope_table(int max_positions, int rot_dim, double base, int scaling, double factor, int original_positions, float *table)
{
    if (max_positions < 1 || max_positions > (1 << 26) || rot_dim < 16 || rot_dim > 1024 || rot_dim % 16)
        return fail(LQ_ERR_INVALID, "bad table: %d positions (1 .. 2^26), rot_dim %d (a multiple of 16 up to 1024)", max_positions, rot_dim);
    if (!(base > 1.0 && base < 1e30)) return fail(LQ_ERR_INVALID, "base must be above 1, got %g", base);
    if (scaling < LQ_ROPE_PLAIN || scaling > LQ_ROPE_YARN) return fail(LQ_ERR_INVALID, "unknown scaling %d", scaling);
    if (scaling != LQ_ROPE_PLAIN && !(factor >= 1.0 && factor < 1e9)) return fail(LQ_ERR_INVALID, "factor must be at least 1, got %g", factor);
    if (scaling == LQ_ROPE_YARN && original_positions < 1) return fail(LQ_ERR_INVALID, "original_positions must be given, got %d", original_positions);
    if (!table) return fail(LQ_ERR_INVALID, "null pointer");
    const int half = rot_dim / 2;
    if (scaling == LQ_ROPE_NTK) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
    // the pairs that turn 32 times and once within the original positions: base^(-2i / rot_dim) original / 2 pi = turns, for i (which may
    // be past the last pair: then none is stretched in full)
    const auto pair_of = [&](double turns) { return rot_dim * std::log(original_positions / (turns * 2.0 * M_PI)) / (2.0 * std::log(base)); };
    double low = 0, high = 0, magnitude = 1.0;
    if (scaling == LQ_ROPE_YARN) {
        low = std::fmax(std::floor(pair_of(32.0)), 0.0);
        high = std::fmin(std::ceil(pair_of(1.0)), rot_dim - 1.0);
        if (high <= low) high = low + 0.001;
        magnitude = 0.1 * std::log(factor) + 1.0;
    }
    double freq[512];
    for (int i = 0; i < half; ++i) {
        freq[i] = std::pow(base, -2.0 * i / rot_dim);
        if (scaling == LQ_ROPE_LINEAR) freq[i] /= factor;
        if (scaling == LQ_ROPE_YARN) {
            const double stretched = std::fmin(std::fmax((i - low) / (high - low), 0.0), 1.0);
            freq[i] *= (1.0 - stretched) + stretched / factor;
        }
    }
    for (int p = 0; p < max_positions; ++p)
        for (int i = 0; i < half; ++i) {
            table[(size_t)p * rot_dim + i] = (float)(std::cos(p * freq[i]) * magnitude);
            table[(size_t)p * rot_dim + half + i] = (float)(std::sin(p * freq[i]) * magnitude);
        }
    return LQ_OK;
}
