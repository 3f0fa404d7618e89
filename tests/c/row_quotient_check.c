/* Exhaustive check of the quotient that a cache row's codes are made of.
 *
 * A row's codes are top x / a (a = max |x|, top = 127 or 448 = 64 * 7) rounded to whole or E4M3 numbers,
 * half to even.  The kernels scale x and a by the power of two that brings a into [1, 2) and form
 * t = top x (exact), r = 1 / a to 2^-22, q0 = RN(t r), q = RN(q0 + RN(t - q0 a) r).
 * For every a = A / 1024, 1024 <= A < 2048, every x = X 2^-k, 1024 <= X < 2048, x <= a, and r = RN(1 / a) and
 * two units in its last place to either side, this program checks that q is RN(t / a), and that rounding q to
 * the code gives the code of the exact quotient, found in integers.  (BF16 and subnormal FP16 numbers are
 * among these.)  Past k = 10 + 24 all codes are 0.  The row's scale a / top is formed alike, with RN(1 / top).
 */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

/* n / d to the nearest whole number, half to even (n, d > 0). */
static uint64_t round_div(unsigned __int128 n, unsigned __int128 d) {
  const unsigned __int128 w = n / d, r2 = 2 * (n % d);
  return (uint64_t)w + (r2 > d || (r2 == d && (w & 1)));
}

int main(void) {
  long long pairs = 0, mismatches = 0, wrong = 0;
  for (int A = 1024; A < 2048; ++A) {
    const volatile float a = (float)A / 1024.0f;
    const float inv = 1.0f / a;
    for (int e4m3 = 0; e4m3 < 2; ++e4m3) {
      const float top = e4m3 ? 448.0f : 127.0f, c = 1.0f / top;
      const float s0 = a * c, s = fmaf(fmaf(-s0, top, a), c, s0);
      const volatile float want = a / top;
      if (s != want) ++mismatches;
    }
    for (int off = -2; off <= 2; ++off)
    for (int k = 10; k <= 36; ++k) {
      const volatile float r = inv + (float)off * ldexpf(1.0f, -24);   /* 1 / a lies in (1/2, 1] */
      for (int X = 1024; X < 2048; ++X) {
        const float x = ldexpf((float)X, -k);
        if (x > a) break;
        for (int e4m3 = 0; e4m3 < 2; ++e4m3) {
          const float t = x * (e4m3 ? 448.0f : 127.0f);
          const float q0 = t * r;
          const float q = fmaf(fmaf(-q0, a, t), r, q0);
          const volatile float want = t / a;
          ++pairs;
          if (q != want) ++mismatches;
          if (!e4m3) {
            /* 127 X 2^-k / (A 2^-10) */
            const uint64_t code = round_div((unsigned __int128)127 * X << 10, (unsigned __int128)A << k);
            if (code != (uint64_t)rintf(q)) ++wrong;
          } else {
            /* in units of the E4M3 step 2^s of 448 x / a */
            const float y = q;
            int e;
            frexpf(y, &e);
            /* the exact quotient may lie on the other side of a power of two only if q rounded up to it,
             * where both steps give the same code */
            const int s = (e > -5 ? e : -5) - 4;
            unsigned __int128 n = (unsigned __int128)448 * X << 10, d = (unsigned __int128)A << k;
            if (s < 0) n <<= -s; else d <<= s;
            if (round_div(n, d) != (uint64_t)rintf(ldexpf(y, -s))) ++wrong;
          }
        }
      }
    }
  }
  printf("pairs %lld mismatches %lld wrong_codes %lld\n", pairs, mismatches, wrong);
  return (mismatches || wrong) ? 1 : 0;
}
