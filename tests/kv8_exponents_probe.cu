// A tile of the many-rows attention kernel as far as its exponents go, on the host, for tests/test_kv8_exponents.py: the maximum is moved and
// the weights' exponents are made by the kernel's own functions and in its order.
#include "eosq_kv8.cuh"

using namespace eosq;

// scores [rows][128], ks and vlog for every 16 of them; m [rows] before and after; exps [rows][128] of the weights, those that were made before the maximum moved
// rescaled.  Returns how many looks at a score that took, at most.
extern "C" int probe_tile(const float *scores, const float *ks, const float *vlog, int rows, int look, float *m, float *exps) {
    int done = 0, looks = 1;
    bool far = false;
    for (int r = 0; r < rows; ++r) far |= m[r] == -INFINITY || kv8_far(m[r]);
    if (!look && !far) {
        for (; done < 128; done += 64) {
            bool over = false;
            for (int r = 0; r < rows; ++r) {
                float sum = 0.0f;
                for (int j = done; j < done + 64; ++j) {
                    const float e = fmaf(scores[r * 128 + j], ks[j / 16], (vlog[j / 16] + KV8_SHIFT) - m[r]);
                    exps[r * 128 + j] = e;
                    sum += exp2f(e);
                }
                over |= sum > 16384.0f;
            }
            if (over) break;
        }
    }
    if (done == 128) return looks;
    looks += 2;
    bool moved = false;
    float top[32];
    for (int r = 0; r < rows; ++r) {
        top[r] = -INFINITY;
        for (int j = done; j < 128; ++j) top[r] = fmaxf(top[r], fmaf(scores[r * 128 + j], ks[j / 16], vlog[j / 16]));
        moved |= top[r] - m[r] > ((look || far) ? KV8_SLACK : 0.0f);
    }
    for (int r = 0; r < rows; ++r) {
        if (moved) {
            const float to = kv8_moved(m[r], top[r]);
            for (int j = 0; j < done; ++j) exps[r * 128 + j] += m[r] - to;
            m[r] = to;
        }
    }
    for (int r = 0; r < rows; ++r)
        for (int j = done; j < 128; ++j) {
            const float x = scores[r * 128 + j], kf = ks[j / 16], m0 = m[r] == -INFINITY ? 0.0f : m[r];
            exps[r * 128 + j] = kv8_far(m[r]) ? fmaf(fmaf(x, kf, vlog[j / 16]) - m0, 1.0f, KV8_SHIFT) : fmaf(x, kf, vlog[j / 16] + (KV8_SHIFT - m0));
        }
    return looks;
}
