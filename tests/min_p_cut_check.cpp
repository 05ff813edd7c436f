// min-p's cut (csrc/min_p_cut.h), run on the host: it is the smallest float whose weight is min_p or more, and found in 34 questions at most,
// wherever it lies.
// usage: min_p_cut_check <top> <temperature> <min_p>: prints the cut and the questions
//        min_p_cut_check random <trials> <seed>
#include "../paper_2410_11744_amd/csrc/min_p_cut.h"

#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <random>

using namespace dyspec;

static const float kMax = 3.402823466e38f;

// questions; -1: the cut is wrong
static int questions(float top, float temperature, float min_p, float* cut)
{
    const double per_nat = 1.4426950408889634074 / (double)temperature, least = log2((double)min_p);
    int n = 0;
    int* const asked = &n;
    *cut = min_p_cut(top, temperature, per_nat, least, [=] { ++*asked; });
    auto enough = [=](float x) { return ((double)x - (double)top) * per_nat >= least - 0x1p-54; };
    const float below = nextafterf(*cut, -INFINITY);
    const bool right = *cut >= -kMax && *cut <= top && enough(*cut) && (below < -kMax || *cut == 0.0f || !enough(below)) &&
                       (*cut != 0.0f || !enough(-nextafterf(0.0f, 1.0f)));            // (-0 and 0 are one)
    return right ? n : -1;
}

int main(int argc, char** argv)
{
    if (argc != 4) return 2;
    float cut;
    if (argv[1][0] != 'r') {
        const int n = questions(strtof(argv[1], nullptr), strtof(argv[2], nullptr), strtof(argv[3], nullptr), &cut);
        printf("%a %d\n", (double)cut, n);
        return n < 0 || n > 34;
    }
    std::mt19937 rng((unsigned)atoi(argv[3]));
    auto unit = [&] { return (double)(rng() >> 8) / 16777216.0; };
    int most = 0;
    long asked = 0;
    const int trials = atoi(argv[2]);
    for (int t = 0; t < trials; ++t) {
        float temperature, min_p, top;
        const int kind = (int)(rng() % 4);
        min_p = rng() % 8 ? (float)unit() : rng() % 2 ? 1.0f : (float)pow(2.0, -150.0 * unit());
        if (!(min_p > 0.0f)) min_p = 1.0f;
        temperature = rng() % 4 ? (float)(0.05 + 2.0 * unit()) : (float)pow(10.0, -44.0 + 82.0 * unit());
        if (kind == 0) top = (float)(20.0 * unit() - 10.0);
        else if (kind == 1) top = (float)(pow(10.0, -44.0 + 82.0 * unit()) * (rng() % 2 ? 1 : -1));
        else top = (float)(-(double)temperature * log((double)min_p));       // the cut is next to zero
        if (kind == 3) top = nextafterf(top, rng() % 2 ? kMax : -kMax);
        if (!(fabsf(top) <= kMax)) top = kMax;
        const int n = questions(top, temperature, min_p, &cut);
        if (n < 0 || n > 34) {
            printf("top %a temperature %a min_p %a: cut %a, %d\n", (double)top, (double)temperature, (double)min_p, (double)cut, n);
            return 1;
        }
        most = n > most ? n : most;
        asked += n;
    }
    printf("most %d, mean %.2f\n", most, (double)asked / trials);
    return 0;
}
