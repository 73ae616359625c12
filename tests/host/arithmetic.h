// What the arithmetic stand-ins of arithmetic.cpp can be told.
#pragma once
struct Arithmetic {
    bool groups = false;   // weight gradients that wait for the end of a pass
};
extern Arithmetic arithmetic;
